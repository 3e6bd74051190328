"""Hier-AVG with AdamW as the local step and a batch of its own size for each learner.

Algorithm 1 (Sec. 3.1) leaves the local update open as long as learners average their parameters;
HierAvg takes plain SGD steps on equal batches.  Here the rows of all learners' batches follow
one another (``offsets`` says where each learner's begin), a layer of all learners is one grouped
product, the loss and its gradient are the log probabilities of the labels, and one AdamW step
updates every learner's tensors in the learner-indexed matrix [P, ld] and writes the bf16 weights
that the products read, after each learner's gradients were clipped to a norm where one is given.  The averages are the library's.  The moments stay each learner's own.

``python -m paper_1903_05133_gb300.local_adamw`` trains 16 learners of 3072-512-10 for a few rounds.
"""
from __future__ import annotations

import argparse
from typing import Optional, Sequence

import torch

from .configs import MLP512_P16
from .hier_avg import HierAvg, local_average_buffer, local_global_average_buffer
from .operators import (AdamW, clip_gradients, grouped_product, grouped_product_dw, grouped_product_dx, operator_check,
                        token_logprobs, token_logprobs_backward)


class LocalAdamW:
    """P learners of a ReLU MLP ``dims``: K1 AdamW steps, a local average over clusters of S, K2 times
    a round, then the global average."""

    def __init__(self, P: int, S: int, K1: int, K2: int, lr: float, dims: Sequence[int], bits: int = 8,
                 beta1: float = 0.9, beta2: float = 0.999, decay: float = 0.0, device="cuda",
                 max_norm: Optional[float] = None):
        """max_norm: of each learner's gradients, weights and biases together (None: not clipped)."""
        self.layout = HierAvg(P, S, K1, K2, lr, 1, dims, "fp32")       # the rows of [P, ld]
        self.P, self.S, self.K1, self.K2, self.lr, self.dims = P, S, K1, K2, lr, tuple(dims)
        self.max_norm = max_norm
        self.params = self.layout.new_params(device)
        self.copy = torch.zeros_like(self.params, dtype=torch.bfloat16)
        self.layers = self.layout.unpack(self.params)                  # [(W [P, out, in], b [P, out])]
        self.weights = [w for w, _ in self.layout.unpack(self.copy)]
        kw = dict(bits=bits, beta1=beta1, beta2=beta2)
        self.opt_w = AdamW([w for w, _ in self.layers], copies=self.weights, decay=decay, **kw)
        self.opt_b = AdamW([b for _, b in self.layers], **kw)
        self.t = 0

    def load(self, layers) -> None:
        """Sets every learner's parameters (as HierAvg.pack)."""
        self.params.copy_(self.layout.pack(layers, self.params.device))
        self.copy.copy_(self.params)

    def _here(self):
        """The parameters' GPU as the current one."""
        return torch.cuda.device(self.params.device)

    def step(self, X: torch.Tensor, y: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
        """One AdamW step of every learner on its rows of X [rows, dims[0]] (bf16) and y [rows]: those from
        offsets[j] to offsets[j + 1].  Returns the log probability of each label before the step."""
        h, L = [X], len(self.layers)
        for l, (w, (_, b)) in enumerate(zip(self.weights, self.layers)):
            h.append(grouped_product(h[-1], w, offsets, bias=b, relu=l + 1 < L))
        r = token_logprobs(h[-1], y)
        # the mean over a learner's rows
        learner = torch.searchsorted(offsets[1:], torch.arange(X.shape[0], dtype=torch.int32, device=X.device), right=True)
        rows = (offsets[1:] - offsets[:-1])[learner.clamp(max=self.P - 1)].clamp(min=1)
        dy = token_logprobs_backward(h[-1], y, r.lse, None, -1.0 / rows.float())
        dw, db = [None] * L, [None] * L
        for l in reversed(range(L)):
            dw[l], db[l] = grouped_product_dw(dy, h[l], offsets, bias_grad=True)
            if l:
                dy = grouped_product_dx(dy, self.weights[l], offsets, h=h[l])
        if self.max_norm is not None:
            clip_gradients(dw + db, self.max_norm, learners=self.P)
        self.opt_w.step(dw, lr=self.lr)
        self.opt_b.step(db, lr=self.lr)
        self.t += 1
        return r.logp

    def local_average(self) -> None:
        with self._here():
            local_average_buffer(self.params, self.S)
            self.copy.copy_(self.params)

    def global_average(self) -> None:
        """The last local average of a round and the global one, in one pass."""
        with self._here():
            local_global_average_buffer(self.params, self.S)
            self.copy.copy_(self.params)

    def round(self, batches) -> torch.Tensor:
        """K1 * K2 steps on (X, y, offsets) from the iterator ``batches`` with their averages; the last
        step's log probabilities.  Synchronises at its end, and raises if a bounded wait ran out."""
        batches = iter(batches)
        logp = None
        for b in range(self.K2):
            for _ in range(self.K1):
                logp = self.step(*next(batches))
            if b + 1 < self.K2:
                self.local_average()
        self.global_average()
        with self._here():
            operator_check()
        return logp


def ragged_batches(X: torch.Tensor, y: torch.Tensor, B: int, seed: int = 0):
    """Endless batches of B / 2 to 2 B rows of each learner's data X [P, N, d], y [P, N], one after
    the other, with their offsets."""
    P, N, _ = X.shape
    gen = torch.Generator().manual_seed(seed)
    while True:
        n = torch.randint(max(B // 2, 1), min(2 * B, N) + 1, (P,), generator=gen)
        at = [torch.randperm(N, generator=gen)[:k] for k in n.tolist()]
        rows = torch.cat([j * N + a for j, a in enumerate(at)]).to(X.device)
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]).to(torch.int32).to(X.device)
        yield X.reshape(P * N, -1)[rows], y.reshape(-1)[rows], offsets


def main() -> None:
    from .inputs import initial_layers, learner_data

    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rounds", type=int, default=4)
    ap.add_argument("--lr", type=float, default=1e-3)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--max-norm", type=float, default=None, help="clip each learner's gradients to this norm")
    a = ap.parse_args()
    w = MLP512_P16
    X, y = learner_data(w, device="cuda")
    m = LocalAdamW(w.P, w.S, w.K1, w.K2, a.lr, w.dims, bits=a.bits, max_norm=a.max_norm)
    m.load(initial_layers(w, device="cuda"))
    batches = ragged_batches(X, y, w.B, w.seed)
    for n in range(a.rounds):
        logp = m.round(batches)
        print(f"round {n + 1}: mean cross-entropy of the last step's batches {-logp.mean().item():.4f}")


if __name__ == "__main__":
    main()
