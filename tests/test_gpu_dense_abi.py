"""What the dense operators' header promises beyond what the Python calls use: outputs over inputs, outputs with a
stride of their own, calls from several threads on streams of their own."""
import threading

import pytest

import dense_reference as R
from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu

GAP = 77.0  # what stands between an output's rows


def _t(name):
    import torch

    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _kind(dtype):
    import torch

    from paper_2504_01506_gb300 import _lib

    return {torch.float32: _lib.TYPE_FLOAT, torch.bfloat16: _lib.TYPE_BFLOAT, torch.float16: _lib.TYPE_HALF}[dtype]


def _lib_of(torch):
    from paper_2504_01506_gb300 import _lib

    return _lib.load(), torch.cuda.current_stream().cuda_stream


def _wide(torch, rows, cols, pad, dtype):
    """([rows, cols] of rows that are `pad` wider, all of it GAP; the whole)"""
    whole = torch.full((rows, cols + pad), GAP, dtype=dtype, device="cuda")
    return whole[:, :cols], whole


def _at(t):
    return None if t is None else t.data_ptr()


def _norm(torch, x, w, b, y, stats, eps=1e-5):
    lib, st = _lib_of(torch)
    assert lib.mlkv_layer_norm(_at(x), x.stride(0), _kind(x.dtype), *x.shape, _at(w), _at(b), _kind(w.dtype), eps, _at(y), y.stride(0),
                               _kind(y.dtype), _at(stats), st) == 0


def _norm_backward(torch, dy, x, w, stats, dx, dw, db):
    lib, st = _lib_of(torch)
    size = lib.mlkv_layer_norm_backward_workspace(*x.shape)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    assert lib.mlkv_layer_norm_backward(_at(dy), dy.stride(0), _kind(dy.dtype), _at(x), x.stride(0), _kind(x.dtype), *x.shape, _at(w),
                                        _kind(w.dtype), _at(stats), _at(dx), dx.stride(0), _at(dw), _at(db), ws.data_ptr(), size, st) == 0


@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("rows,dim", [(900, 100), (301, 129), (5003, 24), (40, 2048), (7, 8193), (3, 20000)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_layer_norm_over_its_inputs(rows, dim, pad, dtype):
    torch = torch_cuda()
    dtype = _t(dtype)
    torch.manual_seed(dim + pad)
    x, whole_x = _wide(torch, rows, dim, pad, dtype)
    dy, whole_dy = _wide(torch, rows, dim, pad, dtype)
    x.copy_(torch.randn(rows, dim, device="cuda"))
    dy.copy_(torch.randn(rows, dim, device="cuda"))
    w, b = torch.randn(dim, device="cuda"), torch.randn(dim, device="cuda")
    stats, stats2 = (torch.empty(rows, 2, device="cuda") for _ in range(2))
    y, _ = _wide(torch, rows, dim, pad, dtype)
    dx, _ = _wide(torch, rows, dim, pad, dtype)
    sums = [torch.empty(dim, device="cuda") for _ in range(4)]
    _norm(torch, x, w, b, y, stats)
    _norm_backward(torch, dy, x, w, stats, dx, *sums[:2])
    _norm_backward(torch, dy, x, w, stats, dy, *sums[2:])  # d_dx = d_dy
    _norm(torch, x, w, b, x, stats2)                       # d_y = d_x
    assert torch.equal(x, y) and torch.equal(stats, stats2)
    assert torch.equal(dy, dx) and torch.equal(sums[0], sums[2]) and torch.equal(sums[1], sums[3])
    assert (whole_x[:, dim:] == GAP).all() and (whole_dy[:, dim:] == GAP).all()


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("dim", [64, 100, 777, 9000])
@pytest.mark.parametrize("types", [("fp32", "bf16"), ("fp16", "fp16")])
def test_layer_norm_into_rows_with_gaps(dim, pad, types):
    torch = torch_cuda()
    xt, yt = _t(types[0]), _t(types[1])
    torch.manual_seed(dim)
    x, dy = torch.randn(83, dim, device="cuda").to(xt), torch.randn(83, dim, device="cuda").to(yt)
    w, b = torch.randn(dim, device="cuda"), torch.randn(dim, device="cuda")
    y, whole_y = _wide(torch, 83, dim, pad, yt)
    dx, whole_dx = _wide(torch, 83, dim, pad, xt)
    stats, dw, db = torch.empty(83, 2, device="cuda"), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    _norm(torch, x, w, b, y, stats)
    _norm_backward(torch, dy, x, w, stats, dx, dw, db)
    want, tol = R.layer_norm(x, w, b, 1e-5)[:2]
    R.within(y, want, tol + R.rounding(want.abs() + tol, yt), "y")
    for name, got, (e, t) in zip(("dx", "dweight", "dbias"), (dx, dw, db), R.layer_norm_backward(dy, x, w, 1e-5)):
        R.within(got, e, t + R.rounding(e.abs() + t, got.dtype), name)
    assert (whole_y[:, dim:] == GAP).all() and (whole_dx[:, dim:] == GAP).all()


@pytest.mark.parametrize("pad", [1, 4, 8])
@pytest.mark.parametrize("m,n,k", [(5, 200, 96), (150, 310, 77), (700, 520, 200)])
def test_products_into_rows_with_gaps(m, n, k, pad):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import _lib

    lib, st = _lib_of(torch)
    dtype = torch.bfloat16
    torch.manual_seed(m + pad)
    x, w, b, res, dy = (torch.randn(s, device="cuda").to(dtype) for s in ((m, k), (n, k), (n,), (m, n), (m, n)))
    outs = {name: _wide(torch, *s, pad, dtype) for name, s in dict(y=(m, n), pre=(m, n), dx=(m, k), dweight=(n, k)).items()}
    db = torch.empty(n, dtype=dtype, device="cuda")
    a = _lib.LinearArgs(m=m, n=n, k=k, d_x=_at(x), x_stride=k, d_weight=_at(w), weight_stride=k, d_bias=_at(b), d_residual=_at(res),
                        residual_stride=n, d_dy=_at(dy), dy_stride=n, d_dbias=_at(db), type=_lib.TYPE_BFLOAT, activation=_lib.ACT_SILU)
    for name, (t, _) in outs.items():
        setattr(a, f"d_{name}", _at(t))
        setattr(a, f"{name}_stride", t.stride(0))
    for size, call in ((lib.mlkv_linear_workspace, lib.mlkv_linear), (lib.mlkv_linear_backward_workspace, lib.mlkv_linear_backward)):
        a.workspace_bytes = size(a)
        ws = torch.empty(max(a.workspace_bytes, 1), dtype=torch.uint8, device="cuda")
        a.d_workspace = ws.data_ptr()
        assert call(a, st) == 0
    want, tol, z, tz = R.linear(x, w, b, "silu", res)
    R.within(outs["y"][0], want, tol + R.rounding(want.abs() + tol, dtype), "y")
    R.within(outs["pre"][0], z, tz + R.rounding(z.abs() + tz, dtype), "pre")
    for name, got, (e, t) in zip(("dx", "dweight", "dbias"), (outs["dx"][0], outs["dweight"][0], db), R.linear_backward(dy, x, w, b, "silu", dtype)):
        R.within(got, e, t + R.rounding(e.abs() + t, dtype), name)
    for name, (t, whole) in outs.items():
        assert (whole[:, t.shape[1]:] == GAP).all(), name


@pytest.mark.parametrize("pad", [1, 5, 8])
@pytest.mark.parametrize("v", [13, 1001, 40000])
def test_logits_gradient_into_rows_with_gaps(v, pad):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    lib, st = _lib_of(torch)
    for dtype in (torch.float32, torch.bfloat16):
        torch.manual_seed(v)
        x, t, g = (torch.randn(6, v, device="cuda") * 2).to(dtype), torch.randint(v, (6,), device="cuda"), torch.randn(6, device="cuda")
        r = dense.token_logprobs(x, t)
        dz, whole = _wide(torch, 6, v, pad, dtype)
        assert lib.mlkv_token_logprobs_backward(_at(x), v, _kind(dtype), 6, v, _at(t), 1.0, _at(r.entropy), _at(r.stats), _at(g), None, _at(dz),
                                                dz.stride(0), st) == 0
        want, tol = R.token_logprobs_backward(x, t, 1.0, g, None)
        R.within(dz, want, tol + R.rounding(want.abs() + tol, dtype), "dlogits")
        assert (whole[:, v:] == GAP).all()


class _Never:
    def __getattr__(self, name):
        return lambda *a: NotImplemented


@pytest.mark.parametrize("checked", [False, True])
def test_threads_on_streams_of_their_own(checked, monkeypatch):
    """Calls from four threads, each on its own stream, give what they give one after another (checked: by way of
    ctypes, which lets other threads run meanwhile)."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    if checked:
        monkeypatch.setattr(dense, "_calls", _Never())

    def step(x, w, t):
        h, stats = dense.layer_norm(x, out_dtype=torch.bfloat16, save_stats=True)
        y, pre = dense.linear(h, w, activation="silu", save_pre=True)
        r = dense.token_logprobs(y, t, top=7)
        dz = dense.token_logprobs_backward(y, t, r, r.entropy)
        dh, dw, db = dense.linear_backward(dz, h, w, pre, activation="silu", bias=True)
        return [y, *r, dw, db, *(d for d in dense.layer_norm_backward(dh, x, None, stats) if d is not None)]

    inputs, wants = [], []
    for i, (m, k, n) in enumerate([(300, 520, 1000), (20, 1024, 6144), (4099, 77, 130), (1, 512, 16384)]):
        torch.manual_seed(i)
        inputs.append((torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda").bfloat16(), torch.randint(n, (m,), device="cuda")))
        wants.append(step(*inputs[-1]))
    torch.cuda.synchronize()
    bad = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got = step(*inputs[i])
                    if not all(torch.equal(a, b) for a, b in zip(got, wants[i])):
                        bad.append(i)
        except Exception as e:  # noqa: BLE001
            bad.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(inputs))]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not bad
    dense.sync()
