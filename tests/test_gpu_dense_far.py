"""The gated block, the cross entropy and AdamW where places pass 2^31 values: the far end is as the same values by themselves."""
import pytest

import dense_block_reference as ref
from dense_reference import rounding, within
from gpu_helpers import torch_cuda

pytestmark = [pytest.mark.gpu, pytest.mark.slow]


def _normal(torch, shape, sigma, dtype, seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(0, sigma, generator=g)


def test_gated_block_of_many_rows():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    m, k, f, t = 270_000, 48, 8_008, torch.bfloat16
    assert m * f > 1 << 31
    x, wg, wu, dh = (_normal(torch, s, c, t, i) for i, (s, c) in enumerate((((m, k), 1.0), ((f, k), k ** -0.5), ((f, k), k ** -0.5), ((m, f), 0.5))))
    h, gate, up = dense.gated_linear(x, wg, wu, save_pre=True)
    dx, dwg, _ = dense.gated_linear_backward(dh, x, wg, wu, gate, up)
    dense.sync()
    for a in (0, m - 300):
        some = slice(a, a + 300)
        want, tol, *_ = ref.gated(x[some], wg, wu, "silu", t)
        within(h[some], want, tol, "h")
        w, e = ref.gated_backward(dh[some], x[some], wg, wu, "silu", t)[0]
        within(dx[some], w, e + rounding(w.abs() + e, t), "dx")
    assert bool(dwg.isfinite().all())


def test_cross_entropy_of_a_long_weight():
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    n, k, vocab, t = 5, 8_200, 262_200, torch.bfloat16
    assert vocab * k > 1 << 31
    x, w = _normal(torch, (n, k), 1.0, t, 0), _normal(torch, (vocab, k), 2.0 * k ** -0.5, t, 1)
    targets = torch.tensor([0, vocab - 1, vocab - 2, -1, 131_000], device="cuda")
    d = torch.tensor([1.0, -2.0, 0.5, 1.0, 3.0], device="cuda")
    r = dense.linear_cross_entropy(x, w, targets)
    dx, dw = dense.linear_cross_entropy_backward(d, x, w, targets, r)
    dense.sync()
    z = torch.cat([x.double() @ w[a:a + 20_000].double().T for a in range(0, vocab, 20_000)], 1)
    lse = torch.logsumexp(z, 1)
    want = torch.where(targets < 0, torch.zeros_like(lse), lse - z.gather(1, targets.clamp(min=0)[:, None])[:, 0])
    # a logit's sum of 8,200 products in fp32 (dense_reference), twice, and the sums of the vocabulary
    tol = 2 * (k + 8) * 2.0 ** -23 * float((x.double().abs() @ w[:1000].double().abs().T).max()) * 1.2 + (vocab / 64 + 100) * 2.0 ** -23
    assert float((r.loss - want).abs().max()) <= tol
    # the last tokens' gradients: P^T x
    p = torch.exp(z[:, -64:] - lse[:, None])
    hot = torch.zeros_like(p)
    hot[1, -1] = hot[2, -2] = 1.0
    g = torch.where(targets < 0, torch.zeros_like(d), d).double()[:, None]
    q = g * (p - hot)
    w64 = q.T @ x.double()
    # P rounded to 8 bits, its exponent off by `tol`, then the output's rounding
    e = (q.abs() * (2.0 ** -8 + tol + 2.0 ** -18) + g.abs() * p * tol).T @ x.double().abs()
    within(dw[-64:], w64, e + rounding(w64.abs() + e, t), "dweight")


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_a_long_tensor(bits):
    torch = torch_cuda()
    from paper_2504_01506_gb300 import dense

    n, last = (1 << 31) + (1 << 20) + 77, 1_000
    p, g = _normal(torch, (n,), 0.1, torch.bfloat16, 0), _normal(torch, (n,), 1e-2, torch.bfloat16, 1)
    tail = [p[-last:].clone()], [g[-last:].clone()]
    state = dense.adamw_state([p], bits)
    dense.adamw([p], [g], state, 1, lr=1e-2)
    torch.cuda.synchronize()
    own = dense.adamw_state(tail[0], bits)
    dense.adamw(tail[0], tail[1], own, 1, lr=1e-2)
    assert torch.equal(p[-last:], tail[0][0])  # (the step is of the state before its rounding to codes)
    if bits == 32:
        assert torch.equal(state.m[0][-last:], own.m[0]) and torch.equal(state.v[0][-last:], own.v[0])
    else:
        assert bool((state.scales[0][:, -1] > 0).all()) and bool((state.v[0][-77:].float() > 0).any())
