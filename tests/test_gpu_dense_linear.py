"""The matrix product with bias, activation and residual, and its gradients, against the definition in 64 bits."""
import pytest

import dense_reference as R
from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1), (1, 4096, 512), (2, 8, 8), (3, 17, 33), (16, 128, 64), (17, 100, 100), (26, 1024, 416),
         (33, 257, 129), (64, 64, 64), (65, 300, 200), (127, 48, 1030), (128, 256, 64), (129, 385, 1000), (300, 520, 700),
         (1000, 1001, 777), (512, 2048, 4096), (4099, 130, 70), (2500, 24, 8), (700, 1500, 16)]


def _t(name):
    import torch

    return {"bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _matrix(torch, rows, cols, dtype, gen, sigma=1.0, pad=0, skip=0):
    return (torch.randn((rows, cols + pad), generator=gen, device="cuda") * sigma).to(dtype)[:, skip:skip + cols]


def _run(torch, m, n, k, dtype, act="none", bias=True, res=False, pad=0, skip=0, seed=0):
    from paper_2504_01506_gb300 import dense

    gen = torch.Generator("cuda")
    gen.manual_seed(seed * 7919 + m * 131 + n * 17 + k)
    x = _matrix(torch, m, k, dtype, gen, 1.0, pad, skip)
    w = _matrix(torch, n, k, dtype, gen, max(k, 1) ** -0.5, pad, skip)
    b = _matrix(torch, 1, n, dtype, gen, 0.5)[0] if bias else None
    r = _matrix(torch, m, n, dtype, gen, 1.0, pad, skip) if res else None
    dy = _matrix(torch, m, n, dtype, gen, 1.0, pad, skip)
    y, pre = dense.linear(x, w, b, activation=act, residual=r, save_pre=True)
    want, tol, z, tz = R.linear(x, w, b, act, r)
    R.within(y, want, tol + R.rounding(want.abs() + tol, dtype), "y")
    assert (pre is None) == (act == "none")
    if pre is not None:
        R.within(pre, z, tz + R.rounding(z.abs() + tz, dtype), "pre")
    assert torch.equal(y, dense.linear(x, w, b, activation=act, residual=r))
    got = dense.linear_backward(dy, x, w, pre, activation=act, bias=bias)
    for name, g, (e, t) in zip(("dx", "dweight", "dbias"), got, R.linear_backward(dy, x, w, b, act, dtype)):
        if name == "dbias" and not bias:
            assert g is None
            continue
        assert g.dtype == dtype
        R.within(g, e, t + R.rounding(e.abs() + t, dtype), name)
    for p, q in zip(got, dense.linear_backward(dy, x, w, pre, activation=act, bias=bias)):
        assert p is None or torch.equal(p, q)
    dense.sync()


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_sizes(size, dtype):
    torch = torch_cuda()
    m, n, k = size
    _run(torch, m, n, k, _t(dtype))


@pytest.mark.parametrize("act", ["none", "relu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("bias,res", [(True, True), (False, True), (False, False)])
@pytest.mark.parametrize("size", [(5, 200, 96), (150, 310, 77), (260, 520, 640)], ids=str)
def test_epilogues(act, bias, res, size):
    torch = torch_cuda()
    m, n, k = size
    _run(torch, m, n, k, torch.bfloat16, act, bias, res)
    _run(torch, m, n, k, torch.float16, act, bias, res)


@pytest.mark.parametrize("pad,skip", [(1, 0), (1, 1), (4, 4), (8, 8), (5, 3)])
@pytest.mark.parametrize("size", [(7, 64, 128), (200, 136, 72), (31, 99, 1001)], ids=str)
def test_strides_and_alignment(size, pad, skip):
    torch = torch_cuda()
    m, n, k = size
    _run(torch, m, n, k, torch.bfloat16, "silu", True, True, pad, skip)


@pytest.mark.parametrize("size", [(0, 8, 8), (8, 0, 8), (8, 8, 0), (0, 0, 0), (5, 300, 0), (70, 0, 9)], ids=str)
def test_empty_sizes(size):
    """No rows: zero gradients of weight and bias; no columns of x: y is the epilogue of the bias."""
    torch = torch_cuda()
    m, n, k = size
    _run(torch, m, n, k, torch.bfloat16, "gelu_tanh", True, True)


def test_transposed_expanded_and_unwanted():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x = torch.randn(96, 40, device="cuda").bfloat16().t()
    w = torch.randn(96, 72, device="cuda").bfloat16().t()
    y = dense.linear(x, w)
    assert torch.equal(y, dense.linear(x.contiguous(), w.contiguous()))
    dy = torch.ones(1, 1, device="cuda", dtype=torch.bfloat16).expand(40, 72)
    full = dense.linear_backward(dy, x, w, bias=True)
    want = dense.linear_backward(dy.contiguous(), x.contiguous(), w.contiguous(), bias=True)
    assert all(torch.equal(p, q) for p, q in zip(full, want))
    dx, none, _ = dense.linear_backward(dy, x, w, want_dweight=False)
    assert none is None and torch.equal(dx, full[0])
    none, dw, db = dense.linear_backward(dy, x, w, want_dx=False, bias=True)
    assert none is None and torch.equal(dw, full[1]) and torch.equal(db, full[2])
    assert dense.linear_backward(dy, x, w, want_dx=False, want_dweight=False, bias=True)[:2] == (None, None)


def test_infinities_and_nan():
    """They come out where the arithmetic takes them, and only there."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    torch.manual_seed(1)
    x = torch.randn(140, 80, device="cuda").bfloat16()
    w = torch.randn(150, 80, device="cuda").bfloat16()
    clean = dense.linear(x, w)
    x[3, 5] = float("nan")
    x[130, 7] = float("inf")
    for act in ("none", "relu", "silu", "gelu_tanh"):
        y = dense.linear(x, w, activation=act)
        assert y[3].isnan().all()
        z = dense.linear(x, w)
        assert torch.isinf(z[130]).all() and not z[130].isnan().any()
        zero = (y[130] == 0) | (y[130] == -float("inf")) if act != "none" else y[130] < 0
        assert ((y[130] == float("inf")) == (z[130] == float("inf"))).all() and zero[z[130] < 0].all()
    keep = torch.ones(140, dtype=torch.bool)
    keep[[3, 130]] = False
    assert torch.equal(dense.linear(x, w)[keep.cuda()], clean[keep.cuda()])


def test_gradients_against_differences():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    torch.manual_seed(2)
    for act in ("gelu_tanh", "silu"):
        x, w, b, dy = (torch.randn(s, device="cuda").bfloat16() for s in ((21, 40), (37, 40), (37,), (21, 37)))
        _, pre = dense.linear(x, w, b, activation=act, save_pre=True)
        got = dense.linear_backward(dy, x, w, pre, activation=act, bias=True)
        tols = [t + R.rounding(e.abs() + t, torch.bfloat16) for e, t in R.linear_backward(dy, x, w, b, act, torch.bfloat16)]
        at = [t.double() for t in (x, w, b)]
        f = lambda x, w, b: (R.act(x @ w.T + b, act) * dy.double()).sum()  # noqa: E731
        e = 1e-5
        for i in range(3):
            for _ in range(3):
                v = torch.randn_like(at[i])
                up, down = list(at), list(at)
                up[i], down[i] = at[i] + e * v, at[i] - e * v
                slope = (f(*up) - f(*down)) / (2 * e)
                assert abs((got[i].double() * v).sum() - slope) <= (v.abs() * tols[i]).sum() + 1e-6 * (1 + slope.abs())


def test_on_another_stream_and_in_a_graph():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    torch.manual_seed(5)
    x = torch.randn(300, 264, device="cuda").bfloat16()
    w = torch.randn(520, 264, device="cuda").bfloat16()
    dy = torch.randn(300, 520, device="cuda").bfloat16()
    _, pre = dense.linear(x, w, activation="silu", save_pre=True)
    dense.linear_backward(dy, x, w, pre, activation="silu")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, pre = dense.linear(x, w, activation="silu", save_pre=True)
        dx, dw, _ = dense.linear_backward(dy, x, w, pre, activation="silu")
    x.copy_(torch.randn(300, 264, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y2, pre2 = dense.linear(x, w, activation="silu", save_pre=True)
        dx2, dw2, _ = dense.linear_backward(dy, x, w, pre2, activation="silu")
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in ((y, y2), (pre, pre2), (dx, dx2), (dw, dw2)))


def test_more_tiles_than_blocks():
    """Every block takes several tiles, in both accumulators, with and without shares of k."""
    torch = torch_cuda()
    _run(torch, 5000, 2304, 136, torch.bfloat16, "relu", True, True)
    _run(torch, 9000, 264, 72, torch.float16, "none", True, False)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_relu_near_zero(dtype):
    """Sums that cancel to next to nothing beside large ones: their signs, which decide relu's slope, are the exact ones."""
    torch = torch_cuda()
    dtype = _t(dtype)
    from paper_2504_01506_gb300 import dense

    gen = torch.Generator("cuda")
    gen.manual_seed(3)
    m, n, half = 400, 96, 256
    u = _matrix(torch, m, half, dtype, gen)
    w = _matrix(torch, n, half, dtype, gen, 0.06)
    sign = torch.where(torch.rand((m, 1), generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    tiny = (sign * 2.0 ** -20).to(dtype)  # (exact in both types: subnormal in fp16)
    x = torch.cat([u, u, tiny], 1)
    weight = torch.cat([w, w, torch.zeros((n, 1), dtype=w.dtype, device="cuda")], 1)
    for column in (5, 37, 95):  # u v - u v + tiny: z is tiny
        weight[column, half:2 * half] = -w[column]
        weight[column, 2 * half] = 1
    y, pre = dense.linear(x, weight, activation="relu", save_pre=True)
    exact = x.double() @ weight.double().T
    for column in (5, 37, 95):
        assert torch.equal(pre[:, column].double(), exact[:, column])
        assert torch.equal(y[:, column].double(), exact[:, column].clamp(min=0))


@pytest.mark.parametrize("n", [77, 256, 300])
def test_relu_near_zero_at_the_last_columns(n):
    """The same where the last block of columns is not whole, and with a bias."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    gen = torch.Generator("cuda")
    gen.manual_seed(n)
    m, half, dtype = 200, 128, torch.bfloat16
    u, w = _matrix(torch, m, half, dtype, gen), _matrix(torch, n, half, dtype, gen, 0.08)
    bias = _matrix(torch, 1, n, dtype, gen, 0.5)[0]
    sign = torch.where(torch.rand((m, 1), generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    x = torch.cat([u, u, (sign * 2.0 ** -21).to(dtype), torch.ones((m, 1), dtype=dtype, device="cuda")], 1)
    weight = torch.cat([w, w, torch.zeros((n, 2), dtype=dtype, device="cuda")], 1)
    weight[n - 1, half:2 * half] = -w[n - 1]
    weight[n - 1, 2 * half] = 1
    weight[n - 1, 2 * half + 1] = -bias[n - 1]
    y, pre = dense.linear(x, weight, bias, activation="relu", save_pre=True)
    exact = sign[:, 0].double() * 2.0 ** -21
    assert torch.equal(pre[:, n - 1].double(), exact)
    assert torch.equal(y[:, n - 1].double(), exact.clamp(min=0))
