"""The AdamW step against its definition: in 64 bits with derived tolerances, and (8-bit states) bit for bit against the same roundings on the CPU."""
import math

import numpy as np
import pytest

from dense_reference import rounding, within
from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HYPER = dict(lr=3e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)


def _network(torch, sizes, p, g, copy, bits, seed=0, off=0):
    """Tensors of these sizes, `off` values off the start of their memory, with a state that has seen steps."""
    from paper_2504_01506_gb300 import dense

    gen = torch.Generator("cuda")
    gen.manual_seed(seed * 100 + len(sizes))

    def make(n, dtype, sigma):
        x = torch.empty(n + off, device="cuda", dtype=torch.float32).normal_(0, sigma, generator=gen)
        return x.to(dtype)[off:]

    params, grads = [make(n, p, 0.1) for n in sizes], [make(n, g, 1e-2) for n in sizes]
    copies = None if copy is None else [make(n, copy, 1.0) for n in sizes]
    if bits == 32:
        m, v = [make(n, torch.float32, 3e-3) for n in sizes], [make(n, torch.float32, 1e-2) for n in sizes]
        for x in v:
            x.mul_(x)
        return params, grads, copies, dense.AdamWState(m, v, None)
    m = [make(n, torch.float32, 60.0).clamp(-448, 448).to(torch.float8_e4m3fn) for n in sizes]
    v = [make(n, torch.float32, 90.0).abs().clamp(max=448).to(torch.float8_e4m3fn) for n in sizes]
    if off:
        m = [torch.cat([x[:1]] * off + [x]).clone()[off:] if x.numel() else x for x in m]
        v = [torch.cat([x[:1]] * off + [x]).clone()[off:] if x.numel() else x for x in v]
    scales = [torch.full((2, (n + 255) // 256), 2.0 ** -14, device="cuda") for n in sizes]
    return params, grads, copies, dense.AdamWState(m, v, scales)


def _wide(torch, x, scale):
    """8-bit codes as the values they stand for, in 64 bits."""
    return x.double() * scale.double().repeat_interleave(256)[:x.numel()]


def _expected(torch, p, g, m, v, t, dtype, factor=1.0, lr=HYPER["lr"]):
    """(p, m, v) in 64 bits, and their tolerances before a rounding to the parameter's type."""
    (b1, b2), eps, wd = HYPER["betas"], HYPER["eps"], HYPER["weight_decay"]
    p, g = p.double(), g.double() * factor
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    # the factors, their products and the sum are rounded: at most 6 half steps of the terms (8 with g's own square);
    # products below 2^-126 lose up to 2^-149 each
    tm = 7 * U * (b1 * m.abs() + (1 - b1) * g.abs()) + 2.0 ** -147
    tv = 9 * U * v1 + 2.0 ** -147
    root = (v1 / (1 - b2 ** t)).sqrt()
    den = root + eps
    rate = lr / (1 - b1 ** t)
    up = rate * m1 / den
    # the root's error is half of v's; the correction (1 - b^t, by expm1 of a product rounded to 2^-24 of itself), the
    # division (2 units) and the products: 2^-19 of the update holds them all
    tp = 4 * U * (p.abs() + up.abs()) + rate * tm / den + up.abs() * (tv / (2 * v1.clamp(min=1e-300)) + 2.0 ** -19)
    x = p * (1 - lr * wd) - up
    return (x, tp + rounding(x.abs() + tp, dtype)), (m1, tm), (v1, tv)


SIZES = [1, 7, 255, 256, 257, 8192, 8193, 30_001, 100_000, 2]


@pytest.mark.parametrize("p,g,copy", [("float32", "float32", None), ("float32", "bfloat16", "bfloat16"), ("float32", "float16", "float16"),
                                      ("bfloat16", "bfloat16", None), ("float16", "float32", None)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("off", [0, 3], ids=["aligned", "off"])
def test_a_step(p, g, copy, bits, off):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    p, g, copy = getattr(torch, p), getattr(torch, g), copy and getattr(torch, copy)
    params, grads, copies, state = _network(torch, SIZES, p, g, copy, bits, off=off)
    before = [(x.clone(), m.clone(), v.clone()) for x, m, v in zip(params, state.m, state.v)]
    scales = None if bits == 32 else [s.clone() for s in state.scales]
    t = 7
    assert dense.adamw(params, grads, state, t, **HYPER, copies=copies, seed=5) is None
    for i, (x, m, v) in enumerate(before):
        if bits == 32:
            m0, v0 = m.double(), v.double()
        else:
            m0, v0 = _wide(torch, m, scales[i][0]), _wide(torch, v, scales[i][1]) ** 2
        (want, tol), (m1, tm), (v1, tv) = _expected(torch, x, grads[i], m0, v0, t, p)
        within(params[i], want, tol, f"p of {i}")
        if bits == 32:
            within(state.m[i], m1, tm, f"m of {i}")
            within(state.v[i], v1, tv, f"v of {i}")
        else:  # within a code's step: 1/8 of the power of two below, or the least one
            for codes, s, w, e in ((state.m[i], state.scales[i][0], m1, tm), (state.v[i], state.scales[i][1], v1.sqrt(), tv / v1.sqrt().clamp(min=1e-30))):
                s = s.double().repeat_interleave(256)[:w.numel()]
                step = torch.maximum(w.abs() + e, s * 2.0 ** -6) * 0.125
                within(_wide(torch, codes, s[::256].contiguous()), w, step + e, f"codes of {i}")
        if copies is not None:
            assert torch.equal(copies[i], params[i].to(copy))


def _codes_on_cpu(torch, x, hashes):
    """(codes, scales) of fp32 values with the roundings that the header states."""
    n = x.size
    blocks = (n + 255) // 256
    most = np.abs(np.pad(x, (0, blocks * 256 - n)).reshape(blocks, 256)).max(1).view(np.int32)
    power = np.maximum((most >> 23) - 8 + ((most & 0x7FFFFF) > 0x600000), 1)
    scale = (power << 23).astype(np.int32).view(np.float32)
    q = x * (np.float32(1) / scale).repeat(256)[:n]
    step = np.maximum(q.view(np.int32) & 0x7F800000, (127 - 6) << 23).astype(np.int32).view(np.float32) * np.float32(0.125)
    unit = ((hashes >> np.uint32(9)) | np.uint32(0x3F800000)).view(np.float32) - np.float32(1.5)
    return np.clip(q + step * unit, np.float32(-448), np.float32(448)), scale


def _mix(h):
    h ^= h >> 16
    h = h * 0x6A09E667 & 0xFFFFFFFF
    h ^= h >> 15
    h = h * 0xBB67AE85 & 0xFFFFFFFF
    return h ^ h >> 16


@pytest.mark.parametrize("off", [0, 1])
def test_codes_bit_for_bit(off):
    """The 8-bit state of three steps, by the same operations in fp32 on the CPU."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    sizes = [5, 256, 700, 500_000]  # (few bits a gradient: sums meet powers of two, where the rounding of each product tells)
    params, grads, _, state = _network(torch, sizes, torch.float32, torch.bfloat16, None, 8, seed=3, off=off)
    f = np.float32
    for t in (1, 2, 1000):
        m0 = [(m.float().cpu().numpy() * s[0].cpu().numpy().repeat(256)[:m.numel()]) for m, s in zip(state.m, state.scales)]
        r0 = [(v.float().cpu().numpy() * s[1].cpu().numpy().repeat(256)[:v.numel()]) for v, s in zip(state.v, state.scales)]
        dense.adamw(params, grads, state, t, **HYPER, seed=0xFFFFFFFF)
        for i, n in enumerate(sizes):
            g = grads[i].float().cpu().numpy()
            m1 = m0[i] * f(0.9) + g * f(1 - 0.9)
            v1 = r0[i] * r0[i] * f(0.999) + g * g * f(1 - 0.999)
            r1 = np.sqrt(v1)
            key = _mix((_mix((_mix(0xFFFFFFFF) + t) & 0xFFFFFFFF) + i) & 0xFFFFFFFF)
            h = (np.arange(n, dtype=np.uint64) * 0x9E3779B9 + key).astype(np.uint32)
            h ^= h >> np.uint32(15)
            qm, sm = _codes_on_cpu(torch, m1, h * np.uint32(0x6A09E667))
            qr, sr = _codes_on_cpu(torch, r1, h * np.uint32(0xBB67AE85))
            qr = np.where(r1 > 0, np.maximum(qr, f(2.0 ** -9)), f(0))
            for got, want in ((state.m[i], qm), (state.v[i], qr)):
                assert torch.equal(got.cpu().view(torch.uint8), torch.from_numpy(want).to(torch.float8_e4m3fn).view(torch.uint8)), (t, i)
            assert np.array_equal(state.scales[i].cpu().numpy(), np.stack([sm, sr])), (t, i)


def test_codes_have_the_value_as_their_mean():
    """Steps without gradients: sqrt(v) decays by sqrt(b2) a step, which to the nearest code it never would."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    n, steps = 1 << 16, 400
    p = [torch.zeros(n, device="cuda")]
    state = dense.adamw_state(p, 8)
    g = torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) + 0.5
    dense.adamw(p, [g], state, 1, **HYPER)
    for t in range(2, steps + 2):
        dense.adamw(p, [torch.zeros_like(g)], state, t, **HYPER)
    want = (g.double() * math.sqrt(1 - 0.999) * 0.999 ** (steps / 2))
    got = _wide(torch, state.v[0], state.scales[0][1])
    # a step's rounding has a standard deviation of at most half a code's step, 1/16 of the value; over `steps` steps that decay
    # slowly, and over n values whose hashes differ: 6 deviations of the mean of got / want
    off = float((got / want).mean()) - 1
    assert abs(off) < 6 * (1 / 16) * math.sqrt(steps / n) + 2.0 ** -8, off


def test_steps_repeat_and_seeds_differ():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    made = []
    for seed, step in ((1, 3), (1, 3), (2, 3), (1, 4)):
        params, grads, _, state = _network(torch, [4096, 33], torch.float32, torch.float32, None, 8)
        dense.adamw(params, grads, state, step, **HYPER, seed=seed)
        made.append(torch.cat([x.view(torch.uint8) for x in state.m + state.v]))
    assert torch.equal(made[0], made[1])
    assert not torch.equal(made[0], made[2]) and not torch.equal(made[0], made[3])


@pytest.mark.parametrize("bits", [32, 8])
def test_step_rate_and_factor_on_the_device(bits):
    """As by value, to the roundings of the corrections; captured and replayed they are read anew."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    sizes = [300, 70_000]
    params, grads, _, state = _network(torch, sizes, torch.float32, torch.bfloat16, None, bits)
    clone = lambda xs: None if xs is None else [x.clone() for x in xs]  # noqa: E731
    ps, st = clone(params), dense.AdamWState(*(clone(x) for x in state))
    step, lr, factor = torch.tensor([0], device="cuda"), torch.tensor([1.0], device="cuda"), torch.tensor([2.0], device="cuda")
    kw = {k: v for k, v in HYPER.items() if k != "lr"}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step += 1
            dense.adamw(ps, grads, st, step, lr=lr, grad_scale=factor, **kw)
    torch.cuda.current_stream().wait_stream(side)
    for t in range(1, 4):
        lr.fill_(1e-3 * t)
        factor.fill_(0.5 * t)
        graph.replay()
        m0 = [m.double() if bits == 32 else _wide(torch, m, s[0]) for m, s in zip(state.m, state.scales or state.m)]
        v0 = [v.double() if bits == 32 else _wide(torch, v, s[1]) ** 2 for v, s in zip(state.v, state.scales or state.v)]
        want = [_expected(torch, p, g, m, v, t, p.dtype, 0.5 * t, 1e-3 * t) for p, g, m, v in zip(params, grads, m0, v0)]
        dense.adamw(params, [g.float() * (0.5 * t) for g in grads], state, t, lr=1e-3 * t, **kw)
        assert int(step) == t
        for i in range(len(sizes)):
            for p in (params[i], ps[i]):
                within(p, want[i][0][0], want[i][0][1], f"p of {i} at {t}")
            assert torch.equal(st.m[i].view(torch.uint8), state.m[i].view(torch.uint8))
            assert torch.equal(st.v[i].view(torch.uint8), state.v[i].view(torch.uint8))
            params[i].copy_(ps[i])


@pytest.mark.parametrize("bits", [32, 8])
def test_values_that_are_not_finite_stay_their_own(bits):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    params, grads, _, state = _network(torch, [1024], torch.float32, torch.float32, None, bits)
    clean = [x.clone() for x in params], dense.AdamWState(*(None if x is None else [y.clone() for y in x] for x in state))
    dense.adamw(clean[0], [g.clone() for g in grads], clean[1], 5, **HYPER)
    bad = [3, 300, 301, 1023]
    grads[0][bad] = torch.tensor([math.nan, math.inf, -math.inf, 3e38], device="cuda")
    dense.adamw(params, grads, state, 5, **HYPER)
    ok = torch.ones(1024, dtype=torch.bool, device="cuda")
    ok[bad] = False
    assert torch.equal(params[0][ok], clean[0][0][ok])
    assert params[0][bad[0]].isnan()
    if bits == 32:
        assert torch.equal(state.m[0][ok], clean[1].m[0][ok]) and torch.equal(state.v[0][ok], clean[1].v[0][ok])
        assert state.m[0][3].isnan() and state.m[0][300] == math.inf and state.v[0][1023] == math.inf
    else:
        m = _wide(torch, state.m[0], state.scales[0][0])
        assert bool(m[[3, 300, 301]].isnan().all()) and bool(m[ok].isfinite().all())
        assert bool(_wide(torch, state.v[0], state.scales[0][1])[bad].isnan().all())
        # blocks 0 and 1 hold others of their size: their largest finite value, and so their codes, are the clean ones'
        same = ok[:256]
        assert torch.equal(state.m[0][:256].view(torch.uint8)[same] == 0x7F, torch.zeros(255, dtype=torch.bool, device="cuda"))


def test_the_smallest_and_largest_values_of_a_block():
    """Zeros, values next to the least of fp32 and to the largest: codes stay finite, a root above 0 stays above 0."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    for scale in (0.0, 1e-44, 1e-38, 1e-20, 1.0, 1e18):
        g = torch.logspace(-12, 0, 512, device="cuda") * scale
        p = [torch.zeros(512, device="cuda")]
        state = dense.adamw_state(p, 8)
        dense.adamw(p, [g], state, 1, lr=1e-3, weight_decay=0.0)
        assert bool(p[0].isfinite().all()) and float(p[0].abs().max()) <= 1.001e-3
        r = _wide(torch, state.v[0], state.scales[0][1])
        assert bool(r.isfinite().all()) and bool((r >= 0).all())
        v = ((g * g) * torch.tensor(1 - 0.999, device="cuda"))
        assert torch.equal(r > 0, v > 0)


def test_empty_tensors_and_missing_gradients():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    p = [torch.ones(0, device="cuda"), torch.ones(3, 5, device="cuda"), torch.ones(7, device="cuda")]
    g = [torch.ones(0, device="cuda"), None, torch.ones(7, device="cuda")]
    state = dense.adamw_state(p)
    dense.adamw(p, g, state, 1, lr=0.1, weight_decay=0.0)
    assert bool((p[1] == 1).all()) and bool((state.m[1] == 0).all())
    assert torch.allclose(p[2], torch.full_like(p[2], 0.9), atol=1e-6)
    dense.adamw([], [], dense.adamw_state([]), 1, lr=0.1)


def test_more_tensors_than_one_launch_takes():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    p = [torch.full((n % 5 + 1,), float(n), device="cuda") for n in range(1000)]
    g = [torch.full_like(x, 1.0) for x in p]
    dense.adamw(p, g, dense.adamw_state(p), 1, lr=0.5, weight_decay=0.0)
    for n, x in enumerate(p):
        assert torch.allclose(x, torch.full_like(x, n - 0.5), atol=1e-4), n


def test_gradients_with_other_strides_and_another_stream():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    p, g = torch.randn(64, 48, device="cuda"), torch.randn(48, 64, device="cuda")
    a, b = [p.clone()], [p.clone()]
    dense.adamw(a, [g.t()], dense.adamw_state(a), 1, lr=1e-2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dense.adamw(tuple(b), (g.t().contiguous(),), dense.adamw_state(b), 1, lr=1e-2)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a[0], b[0])


class _Never:
    def __getattr__(self, name):
        return lambda *a: NotImplemented


@pytest.mark.parametrize("bits", [32, 8])
def test_same_as_the_checked_call(bits, monkeypatch):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    def run():
        params, grads, copies, state = _network(torch, [10, 5000], torch.float32, torch.bfloat16, torch.bfloat16, bits)
        grads[0] = None
        copies[1] = None
        dense.adamw(params, grads, state, torch.tensor([3], device="cuda"), **HYPER, grad_scale=torch.tensor(0.5, device="cuda"), copies=copies)
        return [x.view(torch.uint8) for x in params + state.m + state.v + copies[:1]]

    fast = run()
    monkeypatch.setattr(dense, "_calls", _Never())
    for a, b in zip(fast, run()):
        assert torch.equal(a, b)


def test_refusals():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import MLKVError, dense

    p = torch.zeros(8, 8, device="cuda")
    st = dense.adamw_state([p])
    s8 = dense.adamw_state([p], 8)
    ok = dict(lr=0.1)
    for kind, call in (
            (TypeError, lambda: dense.adamw([p.cpu()], [p], st, 1, **ok)), (TypeError, lambda: dense.adamw([p], [p.cpu()], st, 1, **ok)),
            (ValueError, lambda: dense.adamw([p], [p[0]], st, 1, **ok)), (ValueError, lambda: dense.adamw([p], [], st, 1, **ok)),
            (TypeError, lambda: dense.adamw([p.double()], [p], st, 1, **ok)), (TypeError, lambda: dense.adamw([p.t()[:4].t()], [p[:, :4]], st, 1, **ok)),
            (ValueError, lambda: dense.adamw([p], [p], st, 0, **ok)), (ValueError, lambda: dense.adamw([p], [p], st, 1 << 63, **ok)),
            (TypeError, lambda: dense.adamw([p], [p], st, torch.tensor([1.0], device="cuda"), **ok)),
            (TypeError, lambda: dense.adamw([p], [p], st, 1, lr=torch.tensor([1], device="cuda"))),
            (TypeError, lambda: dense.adamw([p], [p], st, 1, grad_scale=torch.ones(2, device="cuda"), **ok)),
            (ValueError, lambda: dense.adamw([p], [p], st, 1, seed=-1, **ok)), (ValueError, lambda: dense.adamw([p], [p], st, 1, seed=1 << 32, **ok)),
            (MLKVError, lambda: dense.adamw([p], [p], st, 1, betas=(1.0, 0.9), **ok)), (MLKVError, lambda: dense.adamw([p], [p], st, 1, eps=-1.0, **ok)),
            (MLKVError, lambda: dense.adamw([p], [p], st, 1, lr=math.nan)),
            (MLKVError, lambda: dense.adamw([p, p], [p, p], dense.adamw_state([p, p]), 1, **ok)),
            (MLKVError, lambda: dense.adamw([p, p[4:]], [p, p[4:]], dense.adamw_state([p, p[4:]]), 1, **ok)),
            (MLKVError, lambda: dense.adamw([p], [p], dense.AdamWState(st.m, st.m, None), 1, **ok)),
            (MLKVError, lambda: dense.adamw([p, p.clone()], [p, p], dense.AdamWState(st.m * 2, [p.clone(), p.clone()], None), 1, **ok)),
            (TypeError, lambda: dense.adamw([p], [p], st, 1, copies=[p], **ok)), (TypeError, lambda: dense.adamw([p.half()], [p], st, 1, copies=[p.half()], **ok)),
            (ValueError, lambda: dense.adamw([p], [p], st, 1, copies=[], **ok)), (TypeError, lambda: dense.adamw([p], [p], dense.AdamWState(s8.m, s8.v, None), 1, **ok)),
            (TypeError, lambda: dense.adamw([p], [p], dense.AdamWState(st.m, st.v, s8.scales), 1, **ok)),
            (ValueError, lambda: dense.adamw_state([p], 16))):
        with pytest.raises(kind):
            call()
    assert not p.any()
