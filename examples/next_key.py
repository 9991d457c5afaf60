"""Trains a small next-key model over an embedding store.

Each sample is a window of keys; the model predicts the key that follows.  What a
key means is held by the store (rows and Adagrad state); the network between its
Get and the apply of its gradients is made of the package's dense operators:

    rows = store.get(keys)                     fp32, one row a key
    h = layer_norm(rows)                       to bf16
    h = linear(window of h) -> GELU            the window's rows side by side
    h = linear(h) + h                          a second layer, with a residual
    z = linear(h, classes)                     a score for every class
    loss = -log probability of the next key    token_logprobs

and their gradients, down to store.apply_grad(keys, ...).  The dense weights are
kept in fp32 and stepped by plain gradient descent; their bf16 copies are what
the products take.  Run: python examples/next_key.py
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_01506_gb300 import EmbeddingStore, dense  # noqa: E402

BF16 = torch.bfloat16


class NextKey:
    """keys (int64 [n, window]) -> scores of `classes` next keys."""

    def __init__(self, window: int, dim: int, hidden: int, classes: int, capacity: int, max_batch: int, lr: float = 0.5,
                 seed: int = 0):
        g = torch.Generator("cuda")
        g.manual_seed(seed)
        normal = lambda *shape, s: torch.randn(shape, generator=g, device="cuda") * s  # noqa: E731
        self.window, self.dim, self.lr = window, dim, lr
        self.store = EmbeddingStore(dim=dim, capacity=capacity, max_batch=max_batch * window, lr=0.05, init_lo=-1.0, init_hi=1.0)
        self.p = {
            "g": torch.ones(dim, device="cuda"), "b": torch.zeros(dim, device="cuda"),
            "w1": normal(hidden, window * dim, s=(window * dim) ** -0.5), "b1": torch.zeros(hidden, device="cuda"),
            "w2": normal(hidden, hidden, s=hidden ** -0.5), "b2": torch.zeros(hidden, device="cuda"),
            "wc": normal(classes, hidden, s=hidden ** -0.5),
        }

    def forward(self, keys: torch.Tensor) -> dict:
        n = keys.shape[0]
        p = {k: v.to(BF16) if k[0] == "w" or k in ("b1", "b2") else v for k, v in self.p.items()}
        s = {"p": p, "keys": keys.reshape(-1)}
        s["rows"] = self.store.get(s["keys"])
        h, s["stats"] = dense.layer_norm(s["rows"], p["g"], p["b"], out_dtype=BF16, save_stats=True)
        s["x"] = h.view(n, self.window * self.dim)
        s["h1"], s["pre1"] = dense.linear(s["x"], p["w1"], p["b1"], activation="gelu_tanh", save_pre=True)
        s["h2"], s["pre2"] = dense.linear(s["h1"], p["w2"], p["b2"], activation="gelu_tanh", residual=s["h1"], save_pre=True)
        s["logits"] = dense.linear(s["h2"], p["wc"])
        return s

    def step(self, keys: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """One training step; the mean loss, on the device."""
        s = self.forward(keys)
        p, n = s["p"], keys.shape[0]
        r = dense.token_logprobs(s["logits"], targets)
        dz = dense.token_logprobs_backward(s["logits"], targets, r, torch.full_like(r.logprob, -1.0 / n), in_place=True)
        d = {}
        dh2, d["wc"], _ = dense.linear_backward(dz, s["h2"], p["wc"])
        dh1, d["w2"], d["b2"] = dense.linear_backward(dh2, s["h1"], p["w2"], s["pre2"], activation="gelu_tanh", bias=True)
        dh1 += dh2  # the residual's
        dx, d["w1"], d["b1"] = dense.linear_backward(dh1, s["x"], p["w1"], s["pre1"], activation="gelu_tanh", bias=True)
        drows, d["g"], d["b"] = dense.layer_norm_backward(dx.view(-1, self.dim), s["rows"], p["g"], s["stats"])
        self.store.apply_grad(s["keys"], drows)
        for k, v in d.items():
            self.p[k].add_(v, alpha=-self.lr)
        return -r.logprob.mean()

    def predict(self, keys: torch.Tensor, top: int = 5):
        """The likeliest next classes of each window and their log probabilities, with the entropy."""
        s = self.forward(keys)
        r = dense.token_logprobs(s["logits"], torch.full((keys.shape[0],), -1, device="cuda"), top=top)
        return r.top_ids, r.top_logprobs, r.entropy


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
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--keys", type=int, default=64)
    ap.add_argument("--classes", type=int, default=50)
    a = ap.parse_args(argv)
    m = NextKey(a.window, a.dim, a.hidden, a.classes, capacity=max(a.keys, 1024), max_batch=a.samples)
    losses = []
    for t in range(a.steps):
        loss = m.step(*batch(a.samples, a.window, a.keys, a.classes, t))
        if t % 50 == 0 or t == a.steps - 1:
            losses.append(float(loss))
            print(f"step {t:4d}  loss {losses[-1]:.4f}", flush=True)
    dense.sync()
    keys, targets = batch(a.samples, a.window, a.keys, a.classes, 1 << 20)
    ids, _, entropy = m.predict(keys)
    hits = float((ids[:, 0] == targets).float().mean())
    print(f"held-out: first choice right {hits:.3f}, mean entropy {float(entropy.mean()):.3f} nats")
    return losses, hits


if __name__ == "__main__":
    main()
