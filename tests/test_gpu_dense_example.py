"""The next-key example: its step's gradients are those of the same model in plain torch, and it learns."""
import importlib.util
import math
import os

import pytest

from gpu_helpers import torch_cuda

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "next_key.py")


def _example():
    spec = importlib.util.spec_from_file_location("next_key", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_a_step_is_the_models_gradient():
    """Weights after one step against autograd in fp32 on the same bf16 weights, within what bf16 activations round
    (2^-8 of each factor along a chain of at most 12 of them, of the gradient's norm)."""
    torch = torch_cuda()
    ex = _example()
    m = ex.NextKey(window=3, dim=20, hidden=72, classes=33, capacity=500, max_batch=256)
    keys, targets = ex.batch(256, 3, 90, 33, seed=5)
    rows = m.store.get(keys.reshape(-1)).clone().requires_grad_()
    before = {k: v.clone() for k, v in m.p.items()}
    w = {k: (v.bfloat16().float() if k[0] == "w" or k in ("b1", "b2") else v).clone().requires_grad_() for k, v in m.p.items()}
    F = torch.nn.functional
    h = F.layer_norm(rows, (20,), w["g"], w["b"]).view(256, 60)
    h1 = F.gelu(F.linear(h, w["w1"], w["b1"]), approximate="tanh")
    h2 = F.gelu(F.linear(h1, w["w2"], w["b2"]), approximate="tanh") + h1
    want = F.cross_entropy(F.linear(h2, w["wc"]), targets)
    want.backward()
    _, state = m.store.export(keys.reshape(-1).unique())
    assert float(state.abs().max()) == 0
    loss = m.step(keys, targets)
    want = float(want.detach())
    assert abs(float(loss) - want) <= 12 * 2.0 ** -8 * want
    for k in m.p:
        got = (before[k] - m.p[k]) / m.lr
        assert float((got - w[k].grad).norm()) <= 12 * 2.0 ** -8 * float(w[k].grad.norm()), k
    # the store's state: the square of each distinct key's summed gradient
    uniq, inverse = keys.reshape(-1).unique(return_inverse=True)
    g = torch.zeros(uniq.numel(), 20, device="cuda").index_add_(0, inverse, rows.grad)
    _, state = m.store.export(uniq)
    assert float((state.sqrt() - g.abs()).norm()) <= 12 * 2.0 ** -8 * float(g.norm())


def test_it_learns():
    torch_cuda()
    losses, hits = _example().main(["--steps", "301"])
    assert abs(losses[0] - math.log(50)) < 1.0  # an untrained model: about uniform over 50 classes
    assert losses[-1] < 0.25 * losses[0]
    assert hits > 0.5  # 25 times chance
