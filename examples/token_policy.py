"""A policy over a vocabulary of rewrite rules, trained with the library's operators.

The policy sees the rules applied so far (up to `length` of them, padded with -1) and gives a distribution over the next: an
embedding per rule and place, their sum, one hidden layer, logits. One training step runs, in this order,

  embedding -> segment_sum -> two products -> token_logp -> token_logp_backward -> products -> embedding_backward -> muon_step

with the matrices of the two layers and their gradients in flat vectors, as the library keeps an encoder's weights, and plain
gradient steps on the table. The synthetic histories are followed by a rule that depends on their first one.

  python examples/token_policy.py [--steps 80]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2304_14698_amd as xrl  # noqa: E402


class TokenPolicy:
    def __init__(self, rules=150, length=8, dim=64, hidden=256, seed=0):
        model = dict(n_op_types=rules, n_node_dense=0, d_edge=4, d_global=0, hidden=64, rounds=0)
        self.ops = xrl.Encoder(model, np.zeros(xrl.weight_count(model), np.float32))
        self.rules, self.length, self.dim = rules, length, dim
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.matrices = np.array([(0, dim, hidden), (dim * hidden, hidden, rules)])
        n = dim * hidden + hidden * rules
        self.weights = torch.cat([(torch.randn(r, c, generator=g, device="cuda") * (2.0 / r) ** 0.5).flatten()
                                  for _, r, c in self.matrices.tolist()])
        self.grads, self.momentum = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
        self.table = torch.randn(rules * length, dim, generator=g, device="cuda") * (dim * length) ** -0.5
        self.dtable = torch.zeros_like(self.table)

    def views(self, flat):
        return [flat[at:at + r * c].view(r, c) for at, r, c in self.matrices.tolist()]

    def forward(self, history, taken=None, top_k=1):
        """history [n, length] int32, -1: no rule; taken [n] int32 or None."""
        n = history.shape[0]
        place = torch.arange(self.length, device="cuda", dtype=torch.int32) * self.rules
        ids = torch.where(history >= 0, history + place, -1).flatten()
        rows = self.ops.embedding(self.table, ids, scale=self.dim ** 0.5)
        ptr = torch.arange(n + 1, device="cuda", dtype=torch.int32) * self.length
        h0 = self.ops.segment_sum(rows, ptr)
        w1, w2 = self.views(self.weights)
        h1 = torch.relu(h0 @ w1)
        logits = h1 @ w2
        return ids, h0, h1, logits, self.ops.token_logp(logits, taken, top_k=top_k)

    def step(self, history, taken, lr=0.02, table_lr=0.5, entropy_weight=0.001):
        """One step on J = -mean logp(taken) - entropy_weight mean entropy; returns J and the share of best rules that were taken."""
        n = history.shape[0]
        ids, h0, h1, logits, f = self.forward(history, taken)
        each = torch.full((n,), -1.0 / n, device="cuda")
        dlogits = self.ops.token_logp_backward(logits, taken, f, each, entropy_weight * each, out=logits)
        w1, w2 = self.views(self.weights)
        g1, g2 = self.views(self.grads)
        torch.matmul(h1.T, dlogits, out=g2)
        dh1 = (dlogits @ w2.T) * (h1 > 0)
        torch.matmul(h0.T, dh1, out=g1)
        drows = (dh1 @ w1.T).repeat_interleave(self.length, 0)      # the gradient of a sum, at each of its terms
        self.ops.embedding_backward(drows, ids, self.dtable.zero_(), scale=self.dim ** 0.5)
        self.ops.muon_step(self.weights, self.grads, self.momentum, self.matrices, lr=lr)
        self.table.sub_(self.dtable, alpha=table_lr)
        J = -(f["logp"].mean() + entropy_weight * f["entropy"].mean())
        return J, (f["top_ids"][:, 0] == taken).float().mean()


def histories(rng, n, rules, length):
    h = rng.integers(0, rules, (n, length))
    h[np.arange(length) >= rng.integers(1, length + 1, (n, 1))] = -1
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    return t(h), t((7 * h[:, 0] + 3) % rules)


def main(steps=80, n=1024, lr=0.02, table_lr=0.5, verbose=True):
    policy, rng = TokenPolicy(), np.random.Generator(np.random.PCG64(0))
    record = []
    for s in range(steps):
        fall = 1.0 - s / steps
        J, right = policy.step(*histories(rng, n, policy.rules, policy.length), lr=lr * fall, table_lr=table_lr * fall)
        if s % 10 == 0 or s == steps - 1:
            record.append((float(J), float(right)))
            if verbose:
                print(f"step {s:3d}: objective {record[-1][0]:.3f}, best rule right {100 * record[-1][1]:.1f} %", flush=True)
    return record


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=80)
    main(ap.parse_args().steps)
