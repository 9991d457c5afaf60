"""The gated block and its gradients against their definitions in 64 bits."""
import pytest

import dense_block_reference as ref
from dense_reference import act, rounding, within
from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu


def _inputs(torch, m, k, f, dtype, seed=0, pad=0):
    g = torch.Generator("cuda")
    g.manual_seed(seed * 7919 + m * 31 + k * 17 + f)

    def r(rows, cols, sigma):
        return (torch.randn((rows, cols + pad), generator=g, device="cuda") * sigma).to(dtype)[:, :cols]

    return r(m, k, 1.0), r(f, k, max(k, 1) ** -0.5), r(f, k, max(k, 1) ** -0.5), r(m, f, 0.5)


def _check(torch, m, k, f, dtype, name, pad=0):
    from paper_2504_01506_gb300 import dense

    x, wg, wu, dh = _inputs(torch, m, k, f, dtype, pad=pad)
    want, tol, (g, tg), (u, tu) = ref.gated(x, wg, wu, name, dtype)
    h, gate, up = dense.gated_linear(x, wg, wu, activation=name, save_pre=True)
    alone = dense.gated_linear(x, wg, wu, activation=name)
    grads = dense.gated_linear_backward(dh, x, wg, wu, gate, up, activation=name)
    dense.sync()
    within(h, want, tol, "h")
    assert torch.equal(h, alone)
    within(gate, g, tg + rounding(g.abs() + tg, dtype), "gate")
    within(up, u, tu + rounding(u.abs() + tu, dtype), "up")
    for got, (w, t), what in zip(grads, ref.gated_backward(dh, x, wg, wu, name, dtype), ("dx", "dw_gate", "dw_up")):
        assert got.dtype == dtype
        within(got, w, t + rounding(w.abs() + t, dtype), what)
    again = dense.gated_linear_backward(dh, x, wg, wu, gate, up, activation=name)
    for a, b in zip(grads, again):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["none", "relu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("m,k,f", [(1, 64, 64), (17, 200, 130), (150, 96, 200)])
def test_activations_and_types(m, k, f, dtype, name):
    torch = torch_cuda()
    _check(torch, m, k, f, getattr(torch, dtype), name)


# Few rows (1 to 64: a cluster joins shares of k), tiles of every width, shares of k that a second launch adds up,
# pairs of blocks; sizes off 8, off tiles, of one.
SIZES = [(1, 4096, 512), (2, 1000, 1024), (16, 72, 40), (33, 777, 1001), (64, 2048, 96), (64, 64, 10_000), (65, 64, 64), (100, 4096, 40),
         (128, 8192, 64), (129, 1024, 33), (300, 520, 1000), (1000, 64, 24), (515, 77, 1001), (4096, 128, 1000), (2048, 768, 1280),
         (2050, 776, 1300), (1, 1, 1), (3, 7, 5), (70, 1, 1), (200, 8, 300), (1, 256, 12_288), (17, 72, 9_729), (33, 40, 20_003)]


@pytest.mark.parametrize("m,k,f", SIZES)
def test_sizes(m, k, f):
    torch = torch_cuda()
    _check(torch, m, k, f, torch.bfloat16, "silu")


@pytest.mark.parametrize("pad", [1, 8])
@pytest.mark.parametrize("m,k,f", [(5, 96, 64), (200, 96, 72), (600, 1024, 333)])
def test_rows_of_wider_matrices(m, k, f, pad):
    torch = torch_cuda()
    _check(torch, m, k, f, torch.float16, "gelu_tanh", pad=pad)


@pytest.mark.parametrize("m,k,f", [(0, 16, 8), (5, 16, 0), (5, 0, 8), (0, 0, 0), (100, 0, 9)])
def test_empty(m, k, f):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, wg, wu, dh = _inputs(torch, m, k, f, torch.bfloat16)
    h, gate, up = dense.gated_linear(x, wg, wu, save_pre=True)
    dx, dwg, dwu = dense.gated_linear_backward(dh, x, wg, wu, gate, up)
    assert h.shape == (m, f) and dx.shape == (m, k) and dwg.shape == dwu.shape == (f, k)
    for t in (h, gate, up, dx, dwg, dwu):
        assert not t.any()


def test_gradients_not_wanted():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, wg, wu, dh = _inputs(torch, 90, 64, 72, torch.bfloat16)
    _, gate, up = dense.gated_linear(x, wg, wu, save_pre=True)
    both = dense.gated_linear_backward(dh, x, wg, wu, gate, up)
    a = dense.gated_linear_backward(dh, x, wg, wu, gate, up, want_dx=False)
    b = dense.gated_linear_backward(dh, x, wg, wu, gate, up, want_dweight=False)
    assert a[0] is None and b[1] is None and b[2] is None
    assert torch.equal(a[1], both[1]) and torch.equal(a[2], both[2]) and torch.equal(b[0], both[0])


def test_gradients_against_differences():
    """The gradients along a direction, against differences of the definition in 64 bits."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, wg, wu, dh = _inputs(torch, 40, 56, 48, torch.float16, seed=3)
    _, gate, up = dense.gated_linear(x, wg, wu, save_pre=True)
    grads = dense.gated_linear_backward(dh, x, wg, wu, gate, up)
    tols = ref.gated_backward(dh, x, wg, wu, "silu", torch.float16)
    at = [t.double() for t in (x, wg, wu)]
    loss = lambda a, b, c: float((dh.double() * act(a @ b.T, "silu") * (a @ c.T)).sum())  # noqa: E731
    eps = 1e-4
    for i in range(3):
        d = torch.randn(at[i].shape, generator=torch.Generator("cuda").manual_seed(i), dtype=torch.float64, device="cuda")
        up_, down = ([a + s * eps * d if j == i else a for j, a in enumerate(at)] for s in (1, -1))
        diff = (loss(*up_) - loss(*down)) / (2 * eps)
        along = float((grads[i].double() * d).sum())
        want, tol = tols[i]
        # the third derivative's term of a difference: eps^2 times sums of the gradient's size
        allowed = float(((tol + rounding(want.abs() + tol, torch.float16)) * d.abs()).sum()) + 1e-6 * float((want.abs() * d.abs()).sum()) + 1e-6
        assert abs(along - diff) <= allowed, (i, along, diff, allowed)


def test_captured_and_replayed_beside_itself():
    """Two captured graphs, replayed on two streams at once, and calls on a third: each as alone."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    cases = [_inputs(torch, m, 512, 640, torch.bfloat16, seed=m) for m in (3, 500, 900)]

    def step(c):
        x, wg, wu, dh = c
        h, gate, up = dense.gated_linear(x, wg, wu, save_pre=True)
        return (h, *dense.gated_linear_backward(dh, x, wg, wu, gate, up))

    want = [[t.clone() for t in step(c)] for c in cases]
    graphs, outs = [], []
    for c in cases[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(c))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        here = step(cases[2])
        torch.cuda.synchronize()
        for got, w in zip([*outs, here], want):
            for a, b in zip(got, w):
                assert torch.equal(a, b)
    dense.sync()


class _Never:
    def __getattr__(self, name):
        return lambda *a: NotImplemented


def test_same_as_the_checked_calls(monkeypatch):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, wg, wu, dh = _inputs(torch, 37, 40, 24, torch.bfloat16)

    def calls():
        h, gate, up = dense.gated_linear(x, wg, wu, activation="gelu_tanh", save_pre=1)
        return [dense.gated_linear(x, wg, wu.t().contiguous().t()), h, gate, up,
                *dense.gated_linear_backward(dh.t().contiguous().t(), x, wg, wu, gate, up, activation="gelu_tanh"),
                dense.gated_linear_backward(dh, x, wg, wu, gate, up, want_dx=0)[1], dense.gated_linear(x, wg, wu, activation=None)]

    fast = calls()
    monkeypatch.setattr(dense, "_calls", _Never())
    for a, b in zip(fast, calls()):
        assert torch.equal(a, b) and a.stride() == b.stride()


def test_refusals():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, wg, wu, dh = _inputs(torch, 6, 16, 8, torch.bfloat16)
    _, gate, up = dense.gated_linear(x, wg, wu, save_pre=True)
    for kind, call in (
            (TypeError, lambda: dense.gated_linear(x.cpu(), wg, wu)), (TypeError, lambda: dense.gated_linear(x.float(), wg, wu)),
            (TypeError, lambda: dense.gated_linear(x, wg.half(), wu)), (ValueError, lambda: dense.gated_linear(x, wg[:, :8], wu)),
            (ValueError, lambda: dense.gated_linear(x, wg, wu[:4])), (TypeError, lambda: dense.gated_linear(x[0], wg, wu)),
            (ValueError, lambda: dense.gated_linear(x, wg, wu, activation="tanh")),
            (ValueError, lambda: dense.gated_linear_backward(dh[:3], x, wg, wu, gate, up)),
            (ValueError, lambda: dense.gated_linear_backward(dh, x, wg, wu, gate[:, :4], up)),
            (TypeError, lambda: dense.gated_linear_backward(dh, x, wg, wu, gate, up.half())),
            (TypeError, lambda: dense.gated_linear_backward(dh, x, wg, wu, None, up)),
            (RuntimeError, lambda: dense.gated_linear(x, wg, wu, save_pre=torch.ones(2)))):
        with pytest.raises(kind):
            call()


@pytest.mark.parametrize("m,k,f", [(300, 200, 520), (4, 4096, 2048), (8192, 1024, 1280)], ids=["single blocks", "a cluster's shares", "pairs"])
def test_waits_run_out_and_are_told(m, k, f):
    """Operands that never come (mlkv_debug_fail) end the kernel with a status; the next call is right."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import MLKVError, _lib, dense

    x, wg, wu, _ = _inputs(torch, m, k, f, torch.bfloat16)
    want = dense.gated_linear(x, wg, wu)
    dense.sync()
    lib = _lib.load()
    assert lib.mlkv_debug_fail(_lib.FAULT_PRODUCT, 1) == _lib.OK
    dense.gated_linear(x, wg, wu)
    with pytest.raises(MLKVError) as e:
        dense.sync()
    assert e.value.code == _lib.ERR_TIMEOUT
    dense.sync()
    assert torch.equal(dense.gated_linear(x, wg, wu), want)
    dense.sync()
