"""The cross entropy of a linear layer and its gradients against their definitions in 64 bits."""
import math

import pytest

import dense_block_reference as ref
from dense_reference import rounding, within
from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu


def _inputs(torch, n, k, vocab, dtype, seed=0, pad=0, sigma=2.0):
    g = torch.Generator("cuda")
    g.manual_seed(seed * 7919 + n * 31 + k * 17 + vocab)
    x = torch.randn((n, k + pad), generator=g, device="cuda").to(dtype)[:, :k]
    w = (torch.randn((vocab, k + pad), generator=g, device="cuda") * (sigma * k ** -0.5)).to(dtype)[:, :k]
    t = torch.randint(vocab, (n,), generator=g, device="cuda")
    if n > 4:
        t[::5] = -1 - t[::5]
    return x, w, t, torch.randn(n, generator=g, device="cuda")


def _check(torch, n, k, vocab, dtype, scale=1.0, pad=0, sigma=2.0, rows=1 << 14):
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, n, k, vocab, dtype, pad=pad, sigma=sigma)
    r = dense.linear_cross_entropy(x, w, t, scale=scale)
    dx, dw = dense.linear_cross_entropy_backward(d, x, w, t, r, scale=scale)
    dense.sync()
    assert r.loss.dtype == torch.float32 and dx.dtype == dw.dtype == dtype
    for a in range(0, n, rows):
        want, tol, *_ = ref.xent_rows(x[a:a + rows], w, t[a:a + rows], scale)
        within(r.loss[a:a + rows], want, tol, "loss")
    (wx, tx), (ww, tw) = ref.xent_backward(d, x, w, t, scale, dtype, rows)
    within(dx, wx, tx + rounding(wx.abs() + tx, dtype), "dx")
    within(dw, ww, tw + rounding(ww.abs() + tw, dtype), "dweight")
    again = dense.linear_cross_entropy(x, w, t, scale=scale)
    assert torch.equal(again.loss, r.loss) and torch.equal(again.stats, r.stats)
    for a, b in zip(dense.linear_cross_entropy_backward(d, x, w, t, r, scale=scale), (dx, dw)):
        assert torch.equal(a, b)


# One row to many; vocabularies of one token, next to tiles of 64, 128 and 256 columns, large; k of one, off 8, off 64; pairs of blocks.
SIZES = [(1, 64, 1), (1, 128, 2), (1, 2048, 20_000), (3, 1, 31), (5, 100, 64), (16, 128, 15_000), (64, 777, 65), (65, 64, 127), (130, 200, 129),
         (100, 16, 257), (128, 1024, 1000), (515, 77, 5001), (1000, 40, 33), (2048, 768, 2560), (2051, 776, 2561), (4099, 33, 300), (2, 8, 262_144)]


@pytest.mark.parametrize("n,k,vocab", SIZES)
def test_sizes(n, k, vocab):
    torch = torch_cuda()
    _check(torch, n, k, vocab, torch.bfloat16)


@pytest.mark.parametrize("n,k,vocab", [(1, 96, 5000), (70, 96, 1000), (600, 1024, 3333)])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_half_precision_rows_of_wider_matrices_and_scales(n, k, vocab, pad):
    torch = torch_cuda()
    _check(torch, n, k, vocab, torch.float16, scale=(0.7, 1.25, 3.0)[pad % 3], pad=pad)


def test_vocabulary_in_pieces():
    """So many rows that the parts of the sums, and the gradients of the logits, are held for some of the vocabulary at a time."""
    torch = torch_cuda()
    _check(torch, 140_000, 24, 4200, torch.bfloat16, rows=20_000)
    _check(torch, 70_001, 200, 9000, torch.bfloat16, rows=10_000)


def test_sharp_and_flat_rows():
    """Logits far apart (probabilities of 0 and 1) and all the same."""
    torch = torch_cuda()
    _check(torch, 200, 64, 700, torch.bfloat16, sigma=40.0)
    _check(torch, 200, 64, 700, torch.float16, sigma=0.0)


def test_losses_that_count_alike():
    """A gradient that 8 bits cannot hold, the same for all rows: what is off is the outputs' own rounding (2^-8 at most, 0.0017 of the
    norm: values spread over a binade), not the gradient's (2^-8 too, in every place alike)."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, _ = _inputs(torch, 600, 96, 3000, torch.bfloat16, sigma=0.5)
    d = torch.full((600,), 1 + 2.0 ** -8 - 2.0 ** -14, device="cuda")
    r = dense.linear_cross_entropy(x, w, t)
    for got, (want, _) in zip(dense.linear_cross_entropy_backward(d, x, w, t, r), ref.xent_backward(d, x, w, t, 1.0, torch.bfloat16)):
        assert float((got.double() - want).norm()) <= 0.002 * float(want.norm())


def test_small_gradients_in_half_precision():
    """Of a mean over many rows without a loss scale: P would be 0 in fp16, were it not held in units of the largest gradient."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 300, 64, 5000, torch.float16)
    r = dense.linear_cross_entropy(x, w, t)
    big = dense.linear_cross_entropy_backward(d, x, w, t, r)
    small = dense.linear_cross_entropy_backward(d * 2.0 ** -10, x, w, t, r)
    for a, b in zip(big, small):
        # the same P, and so the same sums, 2^-10 times: but for the last rounding, in fp16's smallest steps
        assert bool(((a.float() * 2.0 ** -10 - b.float()).abs() <= 2.0 ** -25 + 2.0 ** -10 * 2.0 ** -11 * a.float().abs()).all())


@pytest.mark.parametrize("scale", [2.0 ** -100, 1.7e38])
def test_scales_next_to_their_ends(scale):
    """All logits as one, and none but the largest."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 40, 32, 300, torch.bfloat16)
    z = x.float() @ w.float().T
    t = z.argmax(1)
    r = dense.linear_cross_entropy(x, w, t, scale=scale)
    want = math.log(300) if scale < 1 else 0.0
    assert float((r.loss - want).abs().max()) <= 1e-5
    dx, dw = dense.linear_cross_entropy_backward(d * 1e-30, x, w, t, r, scale=scale)
    assert bool(dx.isfinite().all()) and bool(dw.isfinite().all())


def test_targets_that_are_none_or_not_there():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 40, 32, 90, torch.bfloat16)
    t[:] = -5
    r = dense.linear_cross_entropy(x, w, t)
    assert not r.loss.any()
    dx, dw = dense.linear_cross_entropy_backward(d, x, w, t, r)
    assert not dx.any() and not dw.any()
    t[3] = 90
    t[7] = 89
    r = dense.linear_cross_entropy(x, w, t)
    assert r.loss[3].isnan() and r.loss[7] > 0 and int((r.loss != 0).sum()) == 2
    dx, dw = dense.linear_cross_entropy_backward(d, x, w, t, r)
    assert bool(dx[3].isnan().all()) and bool(dx[7].isfinite().all()) and not dx[8:].any()


def test_values_that_are_not_finite():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 300, 32, 500, torch.bfloat16)
    t.clamp_(min=0)
    clean = dense.linear_cross_entropy(x, w, t).loss
    x[5, 3] = math.nan
    x[9, 3] = math.inf  # a row of +inf and -inf
    r = dense.linear_cross_entropy(x, w, t)
    ok = torch.ones(300, dtype=torch.bool, device="cuda")
    ok[[5, 9]] = False
    assert torch.equal(r.loss[ok], clean[ok]) and bool(r.loss[~ok].isnan().all())
    dx, _ = dense.linear_cross_entropy_backward(d, x, w, t, r)
    assert bool(dx[ok].isfinite().all()) and bool(dx[~ok].isnan().all())
    # gradients that are not finite stay in their rows of dx, and the power of two goes by the others
    x, w, t, d = _inputs(torch, 300, 32, 500, torch.float16)
    t.clamp_(min=0)
    r = dense.linear_cross_entropy(x, w, t)
    want = dense.linear_cross_entropy_backward(d, x, w, t, r)[0]
    most = int(d.abs().argmin())
    d[most] = math.inf
    dx, dw = dense.linear_cross_entropy_backward(d, x, w, t, r)
    keep = torch.arange(300, device="cuda") != most
    assert torch.equal(dx[keep], want[keep]) and not bool(dx[most].isfinite().all()) and not bool(dw.isfinite().all())


def test_all_logits_masked():
    """A row whose every logit is -inf: loss +inf, statistics without NaN, no gradient's P."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t = torch.zeros(3, 8, device="cuda", dtype=torch.bfloat16), torch.ones(70, 8, device="cuda", dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64, device="cuda")
    x[1, 2] = -math.inf
    r = dense.linear_cross_entropy(x, w, t)
    assert r.loss[1] == math.inf and abs(float(r.loss[0]) - math.log(70)) < 1e-5
    w[5:, 2] = 0  # 0 * inf: NaN
    assert dense.linear_cross_entropy(x, w, t).loss[1].isnan()


def test_no_rows():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 0, 16, 50, torch.bfloat16)
    r = dense.linear_cross_entropy(x, w, t)
    dx, dw = dense.linear_cross_entropy_backward(d, x, w, t, r)
    assert r.loss.shape == (0,) and dx.shape == (0, 16) and dw.shape == (50, 16) and not dw.any()


def test_gradients_not_wanted():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 130, 64, 300, torch.bfloat16)
    r = dense.linear_cross_entropy(x, w, t)
    both = dense.linear_cross_entropy_backward(d, x, w, t, r)
    a, b = (dense.linear_cross_entropy_backward(d, x, w, t, r, **k) for k in (dict(want_dx=False), dict(want_dweight=False)))
    assert a[0] is None and b[1] is None and torch.equal(a[1], both[1]) and torch.equal(b[0], both[0])


def test_gradients_against_differences():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 40, 56, 90, torch.float16, seed=3)
    scale = 1.3
    r = dense.linear_cross_entropy(x, w, t, scale=scale)
    grads = dense.linear_cross_entropy_backward(d, x, w, t, r, scale=scale)
    tols = ref.xent_backward(d, x, w, t, scale, torch.float16)
    at = [x.double(), w.double()]
    loss = lambda a, b: float((ref.xent_rows(a, b, t, scale)[0] * d.double()).sum())  # noqa: E731
    eps = 1e-4
    for i in range(2):
        u = torch.randn(at[i].shape, generator=torch.Generator("cuda").manual_seed(i), dtype=torch.float64, device="cuda")
        hi, lo = ([a + s * eps * u if j == i else a for j, a in enumerate(at)] for s in (1, -1))
        diff = (loss(*hi) - loss(*lo)) / (2 * eps)
        along = float((grads[i].double() * u).sum())
        want, tol = tols[i]
        allowed = float(((tol + rounding(want.abs() + tol, torch.float16)) * u.abs()).sum()) + 1e-6 * float((want.abs() * u.abs()).sum()) + 1e-6
        assert abs(along - diff) <= allowed, (i, along, diff, allowed)


def test_as_the_product_and_the_log_probabilities():
    """The loss is what linear and token_logprobs give, but for their logits' rounding."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, _ = _inputs(torch, 500, 128, 3000, torch.float16)
    r = dense.linear_cross_entropy(x, w, t, scale=0.9)
    z = dense.linear(x, w)
    lp = dense.token_logprobs(z, t, scale=0.9)
    most = float(z.abs().max()) * 2.0 ** -11  # of a logit's rounding; the loss takes two, one of them a mean
    assert float((r.loss + lp.logprob).abs().max()) <= 2 * 0.9 * most + 1e-4


def test_captured_and_replayed():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    cases = [_inputs(torch, n, 96, 2000, torch.bfloat16, seed=n) for n in (2, 400, 900)]

    def step(c):
        x, w, t, d = c
        r = dense.linear_cross_entropy(x, w, t)
        return (r.loss, *dense.linear_cross_entropy_backward(d, x, w, t, r))

    want = [[o.clone() for o in step(c)] for c in cases]
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

    x, w, t, d = _inputs(torch, 37, 40, 24, torch.bfloat16)

    def calls():
        r = dense.linear_cross_entropy(x, w, t, scale=0.5)
        return [*r, *dense.linear_cross_entropy(x.t().contiguous().t(), w, t, scale=2), *dense.linear_cross_entropy_backward(d, x, w, t, r, scale=0.5),
                dense.linear_cross_entropy_backward(d, x, w, t, r, scale=0.5, want_dx=0)[1]]

    fast = calls()
    monkeypatch.setattr(dense, "_calls", _Never())
    for a, b in zip(fast, calls()):
        assert torch.equal(a, b) and a.stride() == b.stride()


def test_refusals():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 6, 16, 8, torch.bfloat16)
    r = dense.linear_cross_entropy(x, w, t)
    for kind, call in (
            (TypeError, lambda: dense.linear_cross_entropy(x.cpu(), w, t)), (TypeError, lambda: dense.linear_cross_entropy(x.float(), w, t)),
            (TypeError, lambda: dense.linear_cross_entropy(x, w.half(), t)), (ValueError, lambda: dense.linear_cross_entropy(x, w[:, :8], t)),
            (ValueError, lambda: dense.linear_cross_entropy(x, w[:0], t)), (ValueError, lambda: dense.linear_cross_entropy(x[:, :0], w[:, :0], t)),
            (TypeError, lambda: dense.linear_cross_entropy(x, w, t.int())), (ValueError, lambda: dense.linear_cross_entropy(x, w, t[:3])),
            (ValueError, lambda: dense.linear_cross_entropy(x, w, t, scale=0.0)), (ValueError, lambda: dense.linear_cross_entropy(x, w, t, scale=math.inf)),
            (ValueError, lambda: dense.linear_cross_entropy_backward(d[:2], x, w, t, r)), (TypeError, lambda: dense.linear_cross_entropy_backward(d.half(), x, w, t, r)),
            (RuntimeError, lambda: dense.linear_cross_entropy_backward(d, x, w, t, r, want_dx=torch.ones(2)))):
        with pytest.raises(kind):
            call()


def test_many_steps_in_a_row():
    """Pairs of blocks behind small kernels, again and again, with nothing that waits between them."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, w, t, d = _inputs(torch, 2051, 777, 5001, torch.bfloat16)
    r = dense.linear_cross_entropy(x, w, t)
    want = dense.linear_cross_entropy_backward(d, x, w, t, r)
    for _ in range(20):
        for _ in range(200):
            r = dense.linear_cross_entropy(x, w, t)
            got = dense.linear_cross_entropy_backward(d, x, w, t, r)
        dense.sync()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_waits_run_out_and_are_told():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import MLKVError, _lib, dense

    x, w, t, d = _inputs(torch, 300, 200, 3000, torch.bfloat16)
    r = dense.linear_cross_entropy(x, w, t)
    want = dense.linear_cross_entropy_backward(d, x, w, t, r)
    dense.sync()
    lib = _lib.load()
    for call in (lambda: dense.linear_cross_entropy(x, w, t), lambda: dense.linear_cross_entropy_backward(d, x, w, t, r)):
        assert lib.mlkv_debug_fail(_lib.FAULT_PRODUCT, 1) == _lib.OK
        call()
        with pytest.raises(MLKVError) as e:
            dense.sync()
        assert e.value.code == _lib.ERR_TIMEOUT
        dense.sync()
    assert torch.equal(dense.linear_cross_entropy(x, w, t).loss, r.loss)
    for a, b in zip(dense.linear_cross_entropy_backward(d, x, w, t, r), want):
        assert torch.equal(a, b)
    dense.sync()
