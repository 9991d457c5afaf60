"""The dense operators' calls whose arguments need nothing done give what the checked ones do, and leave the others to them."""
import pytest

from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu


class _Never:
    def __getattr__(self, name):
        return lambda *a: NotImplemented


def _calls(torch, dense, rows, dim):
    g = torch.Generator("cuda")
    g.manual_seed(rows * 31 + dim)
    r = lambda *s, t=torch.bfloat16: torch.randn(s, generator=g, device="cuda").to(t)  # noqa: E731
    x, dy, w, b = r(rows, dim, t=torch.float32), r(rows, dim), r(dim, t=torch.float32), r(dim, t=torch.float32)
    h, wide = r(rows, dim), r(rows, dim + 3)[:, :dim]
    weight, bias, res = r(24, dim), r(24), r(rows, 24)
    z, t = r(rows, 40), torch.randint(40, (rows,), generator=g, device="cuda")
    one = torch.ones(rows, device="cuda")
    stats = dense.layer_norm(x, w, b, save_stats=True)[1]
    lp = dense.token_logprobs(z, t, top=3)
    pre = dense.linear(h, weight, bias, activation="silu", save_pre=True)[1]
    return [
        lambda: dense.layer_norm(x), lambda: dense.layer_norm(x, w, b, out_dtype=torch.float16, save_stats=1),
        lambda: dense.layer_norm(x, None, b, eps=0), lambda: dense.layer_norm(wide, w), lambda: dense.layer_norm(x.t().contiguous().t()),
        lambda: dense.layer_norm_backward(dy, x, w, stats), lambda: dense.layer_norm_backward(dy, x, None, stats, bias=False),
        lambda: dense.linear(h, weight), lambda: dense.linear(wide, weight, bias, activation="silu", residual=res, save_pre=True),
        lambda: dense.linear(h, weight, bias, save_pre=True), lambda: dense.linear(h, weight.t().contiguous().t(), bias),
        lambda: dense.linear_backward(res, h, weight), lambda: dense.linear_backward(res, h, weight, pre, activation="silu", bias=True),
        lambda: dense.linear_backward(res, h, weight, want_dx=False), lambda: dense.linear_backward(res, h, weight, want_dweight=0),
        lambda: dense.token_logprobs(z, t), lambda: dense.token_logprobs(z, t, top=3, scale=0.5), lambda: dense.token_logprobs(z, t, scale=2),
        lambda: dense.token_logprobs_backward(z, t, lp, one), lambda: dense.token_logprobs_backward(z, t, lp, None, one),
        lambda: dense.token_logprobs_backward(z.clone(), t, lp, one, one, in_place=True),
    ]


def _flat(r):
    return [r] if hasattr(r, "dtype") else list(r)


@pytest.mark.parametrize("rows,dim", [(1, 16), (37, 40), (0, 8), (300, 20)])
def test_same_as_the_checked_calls(rows, dim, monkeypatch):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    calls = _calls(torch, dense, rows, dim)
    fast = [_flat(c()) for c in calls]
    assert dense._calls is not None
    monkeypatch.setattr(dense, "_calls", _Never())
    for n, (f, c) in enumerate(zip(fast, calls)):
        s = _flat(c())
        assert len(f) == len(s), n
        for a, b in zip(f, s):
            assert (a is None) == (b is None), n
            if a is not None:
                assert a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride() and a.device == b.device, n
                assert torch.equal(a.view(torch.uint8) if a.numel() else a, b.view(torch.uint8) if b.numel() else b), n


def test_in_place_returns_the_logits():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    z, t = torch.randn(4, 9, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    lp = dense.token_logprobs(z, t)
    assert dense.token_logprobs_backward(z, t, lp, lp.entropy, in_place=True) is z


def test_refusals_are_the_checked_ones():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, h = torch.randn(4, 8, device="cuda"), torch.randn(4, 8, device="cuda", dtype=torch.bfloat16)
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    for kind, call in (
            (TypeError, lambda: dense.layer_norm(x.double())), (TypeError, lambda: dense.layer_norm(x, x[0].double())),
            (TypeError, lambda: dense.layer_norm(x, x[0].cpu())), (ValueError, lambda: dense.layer_norm(x, x[0, :5])),
            (TypeError, lambda: dense.layer_norm(h, out_dtype=torch.float16)), (TypeError, lambda: dense.layer_norm(x, out_dtype=torch.int32)),
            (dense.MLKVError, lambda: dense.layer_norm(x, eps=-1.0)), (TypeError, lambda: dense.layer_norm(x[0])),
            (ValueError, lambda: dense.layer_norm_backward(x[:2], x, None, torch.zeros(4, 2, device="cuda"))),
            (TypeError, lambda: dense.linear(x, x)), (ValueError, lambda: dense.linear(h, h[:, :5])), (TypeError, lambda: dense.linear(h, h.half())),
            (ValueError, lambda: dense.linear(h, h, activation="tanh")), (ValueError, lambda: dense.linear(h, h, h[0, :3])),
            (ValueError, lambda: dense.linear(h, h, residual=h)), (TypeError, lambda: dense.linear_backward(h[:, :4], h, h, activation="relu")),
            (ValueError, lambda: dense.token_logprobs(x, t, top=33)), (ValueError, lambda: dense.token_logprobs(x, t, scale=0.0)),
            (TypeError, lambda: dense.token_logprobs(x, t.int())), (ValueError, lambda: dense.token_logprobs(x, t[:3]))):
        with pytest.raises(kind):
            call()


def test_a_flag_that_is_neither():
    """Something whose truth raises: what it raises, not a result."""
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    x, h = torch.randn(4, 8, device="cuda"), torch.randn(4, 8, device="cuda", dtype=torch.bfloat16)
    t, two = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.ones(2)
    r = dense.token_logprobs(x, t)
    stats = dense.layer_norm(x, save_stats=True)[1]
    for call in (lambda: dense.layer_norm(x, save_stats=two), lambda: dense.layer_norm_backward(x, x, None, stats, bias=two),
                 lambda: dense.linear(h, h, save_pre=two), lambda: dense.linear_backward(h[:, :4], h, h[:4], want_dx=two),
                 lambda: dense.linear_backward(h[:, :4], h, h[:4], bias=two), lambda: dense.linear_backward(h[:, :4], h, h[:4], want_dweight=two),
                 lambda: dense.token_logprobs_backward(x, t, r, r.logprob, in_place=two)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            call()
