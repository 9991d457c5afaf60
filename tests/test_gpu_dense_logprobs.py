"""Token log probabilities, entropy, alternatives and the logits' gradient against the definition in 64 bits."""
import math

import pytest

import dense_reference as R
from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu


def _t(name):
    import torch

    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _check(torch, logits, targets, top, scale=1.0, seed=5):
    from paper_2504_01506_gb300 import dense

    n, v = logits.shape
    r = dense.token_logprobs(logits, targets, top=top, scale=scale)
    lp, ent, every, _ = R.token_logprobs(logits, targets, scale)
    R.within(r.logprob, lp, 2.0 ** -17 * (1 + lp.abs()), "logprob")
    R.within(r.entropy, ent, 2.0 ** -16 * (1 + ent.abs()), "entropy")
    if top:
        ids = R.alternatives(logits, top)
        assert torch.equal(r.top_ids, ids)
        want = torch.where(ids < 0, -math.inf, every.gather(1, ids.clamp(min=0)))
        want = torch.where(every.isnan().any(1, keepdim=True) & (ids >= 0), math.nan, want)
        R.within(r.top_logprobs, want, 2.0 ** -17 * (1 + want.abs()), "alternatives")
    else:
        assert r.top_ids is None and r.top_logprobs is None
    gen = torch.Generator("cuda")
    gen.manual_seed(seed)
    g = torch.randn(n, generator=gen, device="cuda")
    h = torch.randn(n, generator=gen, device="cuda") * 0.3
    for gg, hh in ((g, h), (g, None), (None, h)):
        dz = dense.token_logprobs_backward(logits, targets, r, gg, hh, scale=scale)
        want, tol = R.token_logprobs_backward(logits, targets, scale, gg, hh)
        R.within(dz, want, tol + R.rounding(want.abs() + tol, logits.dtype), "dlogits")
    return r


def _logits(torch, n, v, dtype, seed=0, pad=0, skip=0, sigma=3.0):
    gen = torch.Generator("cuda")
    gen.manual_seed(seed * 7919 + n * 31 + v)
    x = (torch.randn((n, v + pad), generator=gen, device="cuda") * sigma).to(dtype)
    return x[:, skip:skip + v], torch.randint(v, (n,), generator=gen, device="cuda")


@pytest.mark.parametrize("v", [1, 2, 7, 32, 100, 255, 1000, 4099, 8192, 15000, 33333, 131072])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_vocabularies_and_types(v, dtype):
    torch = torch_cuda()
    x, t = _logits(torch, 9, v, _t(dtype))
    _check(torch, x, t, 20)
    _check(torch, x, t, 0, scale=0.6)


@pytest.mark.parametrize("top", [1, 2, 5, 31, 32])
@pytest.mark.parametrize("n,v", [(1, 131072), (3, 50001), (700, 301), (40, 20), (513, 1)])
def test_alternatives(n, v, top):
    torch = torch_cuda()
    x, t = _logits(torch, n, v, torch.bfloat16, seed=top)
    _check(torch, x, t, top, scale=1.25)


@pytest.mark.parametrize("n", [1, 9, 148])
@pytest.mark.parametrize("v,dtype", [(6144, "bf16"), (8192, "fp16"), (12000, "bf16"), (16384, "bf16"), (4100, "fp32"), (8192, "fp32")])
def test_alternatives_of_spans_joined_by_few_threads(v, dtype, n):
    """A row's spans have more alternatives between them than the block that joins them has threads: all of them are
    there before any is looked at, call after call (two inputs in turn, so that what is left of one would show in the other)."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    inputs = [_logits(torch, n, v, _t(dtype), seed=s) for s in (21, 22)]
    for top in (20, 32):
        wants = [R.alternatives(x, top) for x, _ in inputs]
        wrong = torch.zeros((), dtype=torch.int64, device="cuda")
        for _ in range(100):
            for (x, t), want in zip(inputs, wants):
                wrong += (dense.token_logprobs(x, t, top=top).top_ids != want).sum()
        assert int(wrong) == 0
        for x, t in inputs:
            _check(torch, x, t, top)


@pytest.mark.parametrize("pad,skip", [(1, 0), (1, 1), (3, 2), (8, 8), (5, 3)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_strides_and_alignment(pad, skip, dtype):
    torch = torch_cuda()
    for v in (13, 1001, 40000):
        x, t = _logits(torch, 6, v, _t(dtype), pad=pad, skip=skip)
        _check(torch, x, t, 5)


@pytest.mark.parametrize("v", [50, 3000, 70000])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_masks(v, dtype):
    """-inf and the type's lowest value in a third of the places; rows of nothing else; one value left."""
    torch = torch_cuda()
    for low in (-math.inf, torch.finfo(_t(dtype)).min):
        x, t = _logits(torch, 8, v, _t(dtype), seed=2)
        x[torch.rand(x.shape, device="cuda") < 0.33] = low
        x[1] = low
        x[2] = low
        x[2, v // 2] = 1.5
        x[3, :-3] = low
        t[4] = -1
        t[5] = -(2 ** 62)
        t[6] = v
        if low == -math.inf or v > 1000:  # (32 values remain above the lowest: its log probabilities overflow fp32)
            x[3, :40] = 0.25
            for row in (0, 4, 5, 6, 7):
                t[row] = t[row] if int(t[row]) < 0 or int(t[row]) >= v else int(x[row].argmax())
            t[1] = 3
            t[2] = v // 2
            t[3] = 0
            _check(torch, x, t, 20)


@pytest.mark.parametrize("n,v,dtype", [(700, 131072, "bf16"), (2, 600001, "bf16"), (200, 40000, "fp32"), (305, 60000, "fp16")])
def test_spans_that_a_second_kernel_joins(n, v, dtype):
    """Rows in spans that are too many, or too long, for a cluster (the only ones that need working memory)."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import _lib

    lib = _lib.load()
    kind = {"fp32": _lib.TYPE_FLOAT, "bf16": _lib.TYPE_BFLOAT, "fp16": _lib.TYPE_HALF}[dtype]
    for top in (0, 20, 32):
        assert lib.mlkv_token_logprobs_workspace(n, v, kind, top) > 0
        _check(torch, *_logits(torch, n, v, _t(dtype), seed=top), top, scale=0.8)
        x, t = _logits(torch, n, v, _t(dtype), seed=top + 1, pad=3, skip=1)
        ties = torch.arange(v, device="cuda") % 7 < 2
        rows = [  # one after another of the given, as many as there are
            lambda r: r.fill_(-math.inf), lambda r: r[: 2 * v // 3].fill_(-math.inf), lambda r: r[v // 2:v // 2 + 1].fill_(math.nan),
            lambda r: r[5:6].fill_(math.inf), lambda r: r.copy_(ties), lambda r: r[:-3].fill_(-math.inf), lambda r: r.fill_(2.0),
            lambda r: r[v - 2:].fill_(math.nan)]
        for at in range(0, len(rows), min(n, len(rows))):
            y, ty = x.clone(), t.clone()
            for row, change in zip(y, rows[at:at + n]):
                change(row)
            if n > 10:
                ty[8], ty[9] = -1, v
            _check(torch, y, ty, top)


def test_masked_target():
    torch = torch_cuda()
    x, t = _logits(torch, 4, 500, torch.float32)
    x[torch.arange(4), t] = -math.inf
    r = _check(torch, x, t, 3)
    assert (r.logprob == -math.inf).all()


@pytest.mark.parametrize("v", [40, 5000, 60000])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_nan_and_infinity(v, dtype):
    torch = torch_cuda()
    x, t = _logits(torch, 5, v, _t(dtype))
    x[0, v // 3] = math.nan
    x[1, v // 2] = math.inf
    x[2, 1] = x[2, v - 1] = math.nan
    x[2, 5] = math.inf
    x[3] = math.nan
    _check(torch, x, t, 7)


@pytest.mark.parametrize("v", [33, 2048, 16384, 100001])
def test_ties_go_to_the_lowest_index(v):
    torch = torch_cuda()
    gen = torch.Generator("cuda")
    gen.manual_seed(v)
    x = torch.randint(-2, 3, (6, v), generator=gen, device="cuda").to(torch.bfloat16)
    x[0] = 1.0
    x[1] = -0.0
    x[1, ::3] = 0.0
    x[2] = torch.arange(v, device="cuda").to(torch.bfloat16)
    x[3] = -torch.arange(v, device="cuda").to(torch.bfloat16)
    t = torch.randint(v, (6,), generator=gen, device="cuda")
    for top in (1, 20, 32):
        _check(torch, x.clone(), t, top, scale=0.01)


def test_large_values_and_scales():
    torch = torch_cuda()
    x, t = _logits(torch, 7, 3001, torch.float32)
    _check(torch, x + 10000.0, t, 5)
    _check(torch, x * 1e-3, t, 5, scale=50.0)
    _check(torch, x, t, 5, scale=1e-4)
    _check(torch, (x * 3000).half(), t, 5, scale=1e-3)


@pytest.mark.parametrize("n", [0, 1, 2, 1000])
def test_row_counts(n):
    torch = torch_cuda()
    x, t = _logits(torch, n, 777, torch.bfloat16)
    _check(torch, x, t, 4)


def test_in_place_and_transposed():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, t = _logits(torch, 33, 1003, torch.bfloat16, pad=2, skip=1)
    g = torch.randn(33, device="cuda")
    y = x.t().contiguous().t()
    r, ry = dense.token_logprobs(x.contiguous(), t, top=2), dense.token_logprobs(y, t, top=2)
    assert all(torch.equal(p, q) for p, q in zip(r, ry))
    assert torch.equal(dense.token_logprobs_backward(y, t, ry, g), dense.token_logprobs_backward(x.contiguous(), t, r, g))
    with pytest.raises(TypeError):
        dense.token_logprobs_backward(y, t, r, g, in_place=True)
    r = dense.token_logprobs(x, t, top=2)
    want = dense.token_logprobs_backward(x, t, r, g)
    got = dense.token_logprobs_backward(x, t, r, g, in_place=True)
    assert got.data_ptr() == x.data_ptr() and torch.equal(x, want)


def test_gradient_against_differences():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    torch.manual_seed(4)
    x = torch.randn(6, 50, device="cuda")
    x[2, ::4] = -math.inf
    t = torch.tensor([1, 49, 3, -1, 0, 7], device="cuda")
    g, h = torch.randn(6, device="cuda"), torch.randn(6, device="cuda")
    r = dense.token_logprobs(x, t, scale=1.3)
    got = dense.token_logprobs_backward(x, t, r, g, h, scale=1.3).double()
    _, tol = R.token_logprobs_backward(x, t, 1.3, g, h)

    def f(x):
        lp, ent, _, _ = R.token_logprobs(x, t, 1.3)
        return (lp * g.double() + ent * h.double()).sum()

    e = 1e-5
    for _ in range(6):
        v = torch.randn(6, 50, device="cuda", dtype=torch.float64)
        slope = (f(x.double() + e * v) - f(x.double() - e * v)) / (2 * e)
        assert abs((got * v).sum() - slope) <= (v.abs() * (tol + R.rounding(got, torch.float32))).sum() + 1e-6 * (1 + slope.abs())


def test_in_a_graph_and_on_another_stream():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, t = _logits(torch, 5, 70001, torch.float16)
    g = torch.randn(5, device="cuda")
    dense.token_logprobs(x, t, top=8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = dense.token_logprobs(x, t, top=8)
        dz = dense.token_logprobs_backward(x, t, r, g)
    x.copy_(_logits(torch, 5, 70001, torch.float16, seed=9)[0])
    graph.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        r2 = dense.token_logprobs(x, t, top=8)
        dz2 = dense.token_logprobs_backward(x, t, r2, g)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(r, r2)) and torch.equal(dz, dz2)


def test_offsets_past_32_bits():
    """Logits of more than 2^32 bytes and 2^31 values: the last rows."""
    torch = torch_cuda()
    n, v = 16500, 131072
    x = torch.empty((n, v), dtype=torch.bfloat16, device="cuda")
    x[:-2].fill_(-1.0)
    x[-2:] = _logits(torch, 2, v, torch.bfloat16)[0]
    t = torch.zeros(n, dtype=torch.int64, device="cuda")
    from paper_2504_01506_gb300 import dense

    r = dense.token_logprobs(x, t, top=3)
    small = dense.token_logprobs(x[-2:].contiguous(), t[-2:], top=3)
    assert torch.equal(r.top_ids[-2:], small.top_ids)
    R.within(r.logprob[-2:], small.logprob.double(), 2.0 ** -16 * (1 + small.logprob.double().abs()), "logprob")
    g = torch.ones(n, device="cuda")
    dz = dense.token_logprobs_backward(x, t, r, g)
    want, tol = R.token_logprobs_backward(x[-2:], t[-2:], 1.0, g[-2:], None)
    R.within(dz[-2:], want, tol + R.rounding(want.abs() + tol, x.dtype), "dlogits")


@pytest.mark.parametrize("n,v", [(5, 400), (3, 70000), (200, 40000)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_any_finite_scale(n, v, dtype):
    """Up to the largest: all of the weight is at the largest scores, and what the others weigh does not spoil it."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, _ = _logits(torch, n, v, _t(dtype), sigma=0.02)
    t = x.float().argmax(1)
    t[::2] = 7
    g, h = torch.full((n,), 0.5, device="cuda"), torch.full((n,), 0.3, device="cuda")
    for scale in (1e-40, 1e-37, 1e32, 1e37, 2e38, 2.5e38, 3.4e38):
        r = dense.token_logprobs(x, t, top=3, scale=scale)
        lp, ent, every, _ = R.token_logprobs(x, t, scale)
        R.within(r.logprob, lp, 2.0 ** -17 * (1 + lp.abs()), f"logprob, {scale}")
        R.within(r.entropy, ent, 2.0 ** -16 * (1 + ent.abs()), f"entropy, {scale}")
        ids = R.alternatives(x, 3)
        assert torch.equal(r.top_ids, ids)
        want = every.gather(1, ids)
        R.within(r.top_logprobs, want, 2.0 ** -17 * (1 + want.abs()), f"alternatives, {scale}")
        for gg, hh in ((g, h), (g, None), (None, h)):
            dz = dense.token_logprobs_backward(x, t, r, gg, hh, scale=scale)
            want, tol = R.token_logprobs_backward(x, t, scale, gg, hh)
            R.within(dz, want, tol + R.rounding(want.abs() + tol, x.dtype), f"dlogits, {scale}")
