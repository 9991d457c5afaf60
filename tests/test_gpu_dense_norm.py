"""Layer norm and its gradients against the definition in 64 bits."""
import pytest

import dense_reference as R
from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu

TYPES = ["fp32", "bf16", "fp16"]


def _t(name):
    import torch

    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _matrix(torch, rows, dim, dtype, gen, pad=0, skip=0):
    """[rows, dim], every row a slice of one that is `pad` longer, from value `skip` on."""
    x = torch.randn((rows, dim + pad), generator=gen, device="cuda").to(dtype)
    return x[:, skip:skip + dim]


def _run(torch, rows, dim, xt, yt, wt, pad=0, skip=0, weight=True, bias=True, eps=1e-5, shift=0.0, seed=0):
    from paper_2504_01506_gb300 import dense

    gen = torch.Generator("cuda")
    gen.manual_seed(seed + rows * 31 + dim)
    x = _matrix(torch, rows, dim, _t(xt), gen, pad, skip)
    if shift:
        x = (x.float() + shift).to(_t(xt))
    w = (torch.randn(dim, generator=gen, device="cuda") * 0.3 + 1).to(_t(wt)) if weight else None
    b = torch.randn(dim, generator=gen, device="cuda").to(_t(wt)) if bias else None
    dy = _matrix(torch, rows, dim, _t(yt), gen, pad, skip)
    y, stats = dense.layer_norm(x, w, b, eps=eps, out_dtype=_t(yt), save_stats=True)
    want, tol, mu, r, _, rel, dmu = R.layer_norm(x, w, b, eps)
    R.within(y, want, tol + R.rounding(want.abs() + tol, _t(yt)), "y")
    R.within(stats[:, :1], mu, dmu + R.F32 * mu.abs(), "mean")
    R.within(stats[:, 1:], r, (rel + 4 * R.F32) * r, "rstd")
    assert torch.equal(y, dense.layer_norm(x, w, b, eps=eps, out_dtype=_t(yt)))
    dx, dw, db = dense.layer_norm_backward(dy, x, w, stats, bias=bias)
    (ex, tx), (ew, tw), (eb, tb) = R.layer_norm_backward(dy, x, w, eps)
    R.within(dx, ex, tx + R.rounding(ex.abs() + tx, _t(xt)), "dx")
    assert dx.dtype == x.dtype and (dw is None) == (w is None) and (db is None) == (b is None)
    wdt = _t(wt) if weight else torch.float32
    if weight:
        assert dw.dtype == wdt
        R.within(dw, ew, tw + R.rounding(ew.abs() + tw, wdt), "dweight")
    if bias:
        assert db.dtype == wdt
        R.within(db, eb, tb + R.rounding(eb.abs() + tb, wdt), "dbias")
    again = dense.layer_norm_backward(dy, x, w, stats, bias=bias)
    for p, q in zip((dx, dw, db), again):
        assert p is None or torch.equal(p, q)


@pytest.mark.parametrize("dim", [1, 2, 3, 8, 16, 50, 64, 100, 128, 255, 256, 513, 777, 1000, 1024, 2048, 4100, 8192])
@pytest.mark.parametrize("types", [("fp32", "bf16", "fp32"), ("fp32", "fp32", "fp32"), ("bf16", "bf16", "bf16"),
                                   ("fp16", "fp16", "fp32")])
def test_dims_and_types(dim, types):
    torch = torch_cuda()
    _run(torch, 37, dim, *types)


@pytest.mark.parametrize("rows", [0, 1, 2, 7, 8, 9, 31, 1000, 5003])
@pytest.mark.parametrize("dim", [16, 100, 384, 2048])
def test_row_counts(rows, dim):
    torch = torch_cuda()
    _run(torch, rows, dim, "bf16", "bf16", "fp32")
    _run(torch, rows, dim, "fp32", "fp16", "bf16")


@pytest.mark.parametrize("pad,skip", [(1, 0), (1, 1), (2, 2), (4, 4), (5, 0), (8, 8), (8, 3)])
@pytest.mark.parametrize("dim", [64, 100, 129, 1024, 3000])
def test_strides_and_alignment(dim, pad, skip):
    torch = torch_cuda()
    _run(torch, 45, dim, "bf16", "bf16", "bf16", pad, skip)
    _run(torch, 45, dim, "fp32", "bf16", "fp32", pad, skip)


@pytest.mark.parametrize("dim", [8193, 12000, 20001])
@pytest.mark.parametrize("types", [("fp32", "bf16", "fp32"), ("bf16", "bf16", "bf16")])
def test_long_rows(dim, types):
    torch = torch_cuda()
    _run(torch, 11, dim, *types)
    _run(torch, 3, dim, *types, pad=3, skip=1)


@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_without_weight_or_bias(weight, bias):
    torch = torch_cuda()
    _run(torch, 70, 96, "bf16", "bf16", "bf16", weight=weight, bias=bias)
    _run(torch, 70, 20000, "fp32", "fp32", "fp32", weight=weight, bias=bias)


@pytest.mark.parametrize("shift", [10.0, 3000.0])
def test_rows_far_from_zero(shift):
    """The variance is that of the centred values: no cancellation."""
    torch = torch_cuda()
    _run(torch, 50, 500, "fp32", "fp32", "fp32", shift=shift)


def test_constant_rows_and_eps():
    """A row without variance: y is the bias, whatever the row holds."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x = torch.full((5, 64), 3.0, device="cuda")
    b = torch.randn(64, device="cuda")
    assert torch.equal(dense.layer_norm(x, None, b), b.expand(5, 64))
    _run(torch, 20, 64, "fp32", "fp32", "fp32", eps=0.0)
    _run(torch, 20, 64, "fp32", "fp32", "fp32", eps=0.5)


def test_transposed_and_expanded_inputs():
    """Rows that are not contiguous, or one row for all (as the gradient of a sum is)."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x = torch.randn(96, 40, device="cuda").t()
    w = torch.randn(192, device="cuda")[::2]
    y, stats = dense.layer_norm(x, w, None, save_stats=True)
    assert torch.equal(y, dense.layer_norm(x.contiguous(), w.contiguous(), None))
    dy = torch.ones(1, 1, device="cuda").expand(40, 96)
    got = dense.layer_norm_backward(dy, x, w, stats)
    want = dense.layer_norm_backward(dy.contiguous(), x.contiguous(), w.contiguous(), stats)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_gradients_against_differences():
    """Along random directions, central differences of the 64-bit definition."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    torch.manual_seed(3)
    rows, dim, eps, h = 13, 45, 1e-5, 1e-5
    x, w, b, dy = (torch.randn(s, device="cuda") for s in ((rows, dim), (dim,), (dim,), (rows, dim)))
    _, stats = dense.layer_norm(x, w, b, eps=eps, save_stats=True)
    got = dense.layer_norm_backward(dy, x, w, stats)
    tols = [t for _, t in R.layer_norm_backward(dy, x, w, eps)]

    def f(x, w, b):
        mu = x.mean(1, keepdim=True)
        return ((x - mu) / ((x - mu).pow(2).mean(1, keepdim=True) + eps).sqrt() * w + b).mul(dy.double()).sum()

    at = [t.double() for t in (x, w, b)]
    for i in range(3):
        for _ in range(4):
            v = torch.randn_like(at[i])
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            slope = (f(*up) - f(*down)) / (2 * h)
            tol = (v.abs() * (tols[i] + R.rounding(got[i].double(), torch.float32))).sum() + 1e-6 * (1 + slope.abs())
            assert abs((got[i].double() * v).sum() - slope) <= tol


def test_on_another_stream_and_in_a_graph():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x = torch.randn(300, 256, device="cuda")
    w = torch.randn(256, device="cuda")
    want = dense.layer_norm(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = dense.layer_norm(x, w)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, stats = dense.layer_norm(x, w, save_stats=True)
        dx, dw, _ = dense.layer_norm_backward(x, x, w, stats)
    x.copy_(torch.randn_like(x))
    graph.replay()
    y2, stats2 = dense.layer_norm(x, w, save_stats=True)
    dx2, dw2, _ = dense.layer_norm_backward(x, x, w, stats2)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_more_rows_than_blocks_of_both_passes():
    """Many rows of narrow and odd dims: every team takes several."""
    torch = torch_cuda()
    _run(torch, 60_001, 24, "fp32", "bf16", "fp32")
    _run(torch, 20_011, 333, "fp16", "fp16", "fp16")


@pytest.mark.parametrize("rows,dim", [(1, 8), (300, 100), (65536, 2048), (2048, 8192), (5000, 16384), (700, 65536), (12, 2 ** 20 - 1), (10 ** 6, 16384)])
def test_working_memory_of_the_gradients(rows, dim):
    """The sums of as many blocks as run at a time (of long rows: of a few columns' shares), not of every row."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import _lib

    sms = torch.cuda.get_device_properties(0).multi_processor_count
    most = 3 * sms if dim <= 8192 else max(2 * sms * 128 // dim, rows // 256) + 1
    assert 0 <= _lib.load().mlkv_layer_norm_backward_workspace(rows, dim) <= min(rows, most) * 2 * dim * 4
    if rows * dim < 2 ** 28:  # ... and it is enough
        _run(torch, rows, dim, "bf16", "bf16", "fp32")
        _run(torch, rows, dim, "fp32", "bf16", "fp32")


@pytest.mark.parametrize("rows,dim", [(12000, 39040), (24000, 9000)])
def test_column_sums_of_many_long_rows(rows, dim):
    """No sum is a chain of all the rows: a share's at most 256, then the shares', each warp every 32nd."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x = torch.ones(rows, dim, device="cuda")
    x[:, ::2] = -1  # (mean 0, variance 1)
    dy = torch.empty(rows, dim, device="cuda")
    dy[:, : dim // 2], dy[:, dim // 2:] = 0.1, 0.7
    _, stats = dense.layer_norm(x, save_stats=True)
    weight = torch.ones(dim, device="cuda")
    _, dw, db = dense.layer_norm_backward(dy, x, weight, stats)
    eb = rows * dy[0].double()
    ew = eb * x[0].double() / (1 + 1e-5) ** 0.5
    chain = 256 + rows // 256 // 32 + 40
    R.within(db, eb, chain * R.F32 * eb, "dbias")
    R.within(dw, ew, (chain + 16) * R.F32 * ew.abs(), "dweight")


@pytest.mark.parametrize("rows,dim", [(700, 100), (700, 36), (3, 100), (700, 520), (60, 1032), (700, 101), (9, 8200)])
@pytest.mark.parametrize("types", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
def test_infinite_gradients_at_the_last_columns(rows, dim, types):
    """A row's gradient is infinite or NaN where the formula makes it so, column by column; no other row's is."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    gen = torch.Generator("cuda")
    gen.manual_seed(dim)
    x = _matrix(torch, rows, dim, _t(types[0]), gen)
    dy = _matrix(torch, rows, dim, _t(types[1]), gen)
    w = torch.rand(dim, generator=gen, device="cuda") + 0.5
    _, stats = dense.layer_norm(x, w, save_stats=True, out_dtype=_t(types[1]))
    clean = dense.layer_norm_backward(dy, x, w, stats)
    bad = rows // 2
    for column in (dim - 1, dim - 2):
        for value in (float("inf"), -float("inf")):
            d = dy.clone()
            d[bad, column] = value
            dx, dw, db = dense.layer_norm_backward(d, x, w, stats)
            keep = torch.ones(rows, dtype=torch.bool, device="cuda")
            keep[bad] = False
            assert torch.equal(dx[keep], clean[0][keep])
            mu, r = stats[bad, 0].double(), stats[bad, 1].double()
            g, xh = d[bad].double() * w.double(), (x[bad].double() - mu) * r
            want = r * (g - g.mean() - xh * (g * xh).mean())
            assert torch.equal(dx[bad].isnan(), want.isnan()) and torch.equal(dx[bad].isposinf(), want.isposinf())
            assert torch.equal(dx[bad].isneginf(), want.isneginf())
            finite = torch.arange(dim, device="cuda") != column
            assert torch.equal(dw[finite], clean[1][finite]) and torch.equal(db[finite], clean[2][finite])
            assert db[column] == value and dw[column].isinf()
