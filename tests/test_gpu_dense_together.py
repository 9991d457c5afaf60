"""The gated block, the cross entropy and AdamW in one training step over the store: its gradients, and its capture."""
import importlib.util
import os

import pytest

from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_next_key.py")


def _example():
    spec = importlib.util.spec_from_file_location("gated_next_key", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dim,hidden,classes", [(20, 72, 33), (32, 128, 1000)])
def test_gradients_are_the_models(dim, hidden, classes):
    """Against autograd in fp32 on the same bf16 weights, within what bf16 rounds (2^-8 of each factor along a chain of
    at most 12 of them, of the gradient's norm)."""
    torch = torch_cuda()
    ex = _example()
    m = ex.GatedNextKey(window=3, dim=dim, hidden=hidden, classes=classes, capacity=500, max_batch=256)
    keys, targets = ex.batch(256, 3, 90, classes, seed=5)
    rows = m.store.get(keys.reshape(-1)).clone().requires_grad_()
    w = {k: v.float().clone().requires_grad_() for k, v in m.w.items()}
    F = torch.nn.functional
    x = F.layer_norm(rows, (dim,), w["g"], w["b"]).view(256, 3 * dim)
    h = F.silu(F.linear(x, w["gate"])) * F.linear(x, w["up"])
    want = F.cross_entropy(F.linear(F.linear(h, w["down"]) + x, w["classes"]), targets)
    want.backward()
    loss, s = m.loss(keys, targets)
    drows, d = m.gradients(s, targets, torch.full_like(loss, 1 / 256))
    assert abs(float(loss.mean()) - float(want.detach())) <= 12 * 2.0 ** -8 * float(want.detach())
    for k in w:
        assert float((d[k].float() - w[k].grad).norm()) <= 12 * 2.0 ** -8 * float(w[k].grad.norm()), k
    assert float((drows - rows.grad).norm()) <= 12 * 2.0 ** -8 * float(rows.grad.norm())


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_is_the_step(bits):
    """Three steps, each with another batch: replayed, and call by call, bit for bit."""
    torch = torch_cuda()
    ex = _example()
    make = lambda: ex.GatedNextKey(window=3, dim=20, hidden=72, classes=33, capacity=500, max_batch=256, state_bits=bits)  # noqa: E731
    a, b = make(), make()
    batches = [ex.batch(256, 3, 90, 33, seed=t) for t in range(3)]
    for m in (a, b):
        for keys, _ in batches:  # (the same keys in the same order: the same rows)
            m.store.get(keys.reshape(-1))
    for keys, targets in batches:
        want, got = a.step(keys, targets), b.replay(keys, targets)
        assert torch.equal(want, got)
    assert int(a.steps) == int(b.steps) == 3
    for k in a.p:
        assert torch.equal(a.p[k], b.p[k]) and torch.equal(a.w[k], b.w[k]), k
        if a.w[k].dtype == torch.bfloat16:
            assert torch.equal(a.w[k], a.p[k].bfloat16())
    for x, y in zip(a.state.m + a.state.v, b.state.m + b.state.v):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    keys = torch.cat([k.reshape(-1) for k, _ in batches]).unique()
    for x, y in zip(a.store.export(keys), b.store.export(keys)):
        assert torch.equal(x, y)
    ex.dense.sync()


def test_it_runs():
    torch_cuda()
    for bits in ("32", "8"):
        _example().main(["--steps", "3", "--samples", "256", "--state-bits", bits])
