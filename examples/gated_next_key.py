"""Trains a next-key model with a gated block over an embedding store, its step captured into a CUDA graph.

As next_key.py's model, with a gated block between the rows and the classes, a
loss that keeps no scores, and AdamW for the dense weights:

    rows = store.get(keys)                            fp32, one row a key
    x = layer_norm(rows)                              to bf16, the window's rows side by side
    h = act(x Wg^T) * (x Wu^T)                        gated_linear
    y = h Wd^T + x                                    linear
    loss = cross entropy of y Wc^T with the next key  linear_cross_entropy

and their gradients, down to store.apply_grad(keys, ...).  The weights are fp32;
adamw steps them and writes the bf16 copies that the products take.  The number
of the step is on the device, so that the whole step, from the Get to the two
optimizers, is one graph that a new batch is replayed with.

Run: python examples/gated_next_key.py [--state-bits 8]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_01506_gb300 import EmbeddingStore, dense  # noqa: E402

BF16 = torch.bfloat16


class GatedNextKey:
    """keys (int64 [n, window]) -> the loss of the next of `classes` keys."""

    def __init__(self, window: int, dim: int, hidden: int, classes: int, capacity: int, max_batch: int, lr: float = 3e-3,
                 state_bits: int = 32, seed: int = 0):
        g = torch.Generator("cuda")
        g.manual_seed(seed)
        wide = window * dim
        normal = lambda *shape: torch.randn(shape, generator=g, device="cuda") * shape[-1] ** -0.5  # noqa: E731
        self.dim, self.wide, self.lr = dim, wide, lr
        self.store = EmbeddingStore(dim=dim, capacity=capacity, max_batch=max_batch * window, lr=0.05, init_lo=-1.0, init_hi=1.0)
        self.p = {"g": torch.ones(dim, device="cuda"), "b": torch.zeros(dim, device="cuda"), "gate": normal(hidden, wide),
                  "up": normal(hidden, wide), "down": normal(wide, hidden), "classes": normal(classes, wide)}
        self.w = {k: v.to(BF16) if v.dim() == 2 else v for k, v in self.p.items()}  # what the operators take
        self.state = dense.adamw_state(list(self.p.values()), state_bits)
        self.steps = torch.zeros((), dtype=torch.int64, device="cuda")
        self.graph = None

    def loss(self, keys: torch.Tensor, targets: torch.Tensor):
        """(the rows' losses, what the gradients need)"""
        w, s = self.w, {"keys": keys.reshape(-1)}
        s["rows"] = self.store.get(s["keys"])
        x, s["stats"] = dense.layer_norm(s["rows"], w["g"], w["b"], out_dtype=BF16, save_stats=True)
        s["x"] = x.view(-1, self.wide)
        s["h"], s["gate"], s["up"] = dense.gated_linear(s["x"], w["gate"], w["up"], save_pre=True)
        s["y"] = dense.linear(s["h"], w["down"], residual=s["x"])
        s["loss"] = dense.linear_cross_entropy(s["y"], w["classes"], targets)
        return s["loss"].loss, s

    def gradients(self, s: dict, targets: torch.Tensor, dloss: torch.Tensor):
        """(the rows' gradients, those of the dense weights by name)"""
        w, d = self.w, {}
        dy, d["classes"] = dense.linear_cross_entropy_backward(dloss, s["y"], w["classes"], targets, s["loss"])
        dh, d["down"], _ = dense.linear_backward(dy, s["h"], w["down"])
        dx, d["gate"], d["up"] = dense.gated_linear_backward(dh, s["x"], w["gate"], w["up"], s["gate"], s["up"])
        dx += dy  # the residual's
        drows, d["g"], d["b"] = dense.layer_norm_backward(dx.view(-1, self.dim), s["rows"], w["g"], s["stats"])
        return drows, d

    def step(self, keys: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """One training step; the mean loss, on the device."""
        loss, s = self.loss(keys, targets)
        drows, d = self.gradients(s, targets, torch.full_like(loss, 1.0 / loss.numel()))
        self.store.apply_grad(s["keys"], drows)
        self.steps += 1
        copies = [w if w.dtype == BF16 else None for w in self.w.values()]
        dense.adamw(list(self.p.values()), [d[k] for k in self.p], self.state, self.steps, lr=self.lr, weight_decay=0.01, copies=copies)
        return loss.mean()

    def replay(self, keys: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """As step, of a graph that the first call captures (batches of one size)."""
        if self.graph is None:
            self.inputs = keys.clone(), targets.clone()
            self.store.get(keys.reshape(-1))  # (keys that are new are inserted)
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.mean = self.step(*self.inputs)
        self.inputs[0].copy_(keys)
        self.inputs[1].copy_(targets)
        self.graph.replay()
        return self.mean


def batch(n: int, window: int, keys: int, classes: int, seed: int):
    """Windows of skewed keys; the next class is a fixed function of the last two keys."""
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    k = (torch.rand((n, window), generator=g, device="cuda") ** 3 * keys).long()
    return k + (1 << 33), (k[:, -1] * 7 + k[:, -2]) % classes


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--samples", type=int, default=2048)
    ap.add_argument("--window", type=int, default=4)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--keys", type=int, default=64)
    ap.add_argument("--classes", type=int, default=50)
    ap.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    a = ap.parse_args(argv)
    m = GatedNextKey(a.window, a.dim, a.hidden, a.classes, capacity=max(a.keys, 1024), max_batch=a.samples, state_bits=a.state_bits)
    for t in range(a.steps):
        loss = m.replay(*batch(a.samples, a.window, a.keys, a.classes, t))
        if t % 50 == 0 or t == a.steps - 1:
            print(f"step {t:4d}  loss {float(loss):.4f}", flush=True)
    dense.sync()
    keys, targets = batch(a.samples, a.window, a.keys, a.classes, 1 << 20)
    print(f"held-out loss {float(m.loss(keys, targets)[0].mean()):.4f}")


if __name__ == "__main__":
    main()
