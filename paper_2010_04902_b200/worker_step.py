"""A small language model trained the ByzShield way: K = 15 workers compute file gradients, some of them lie, the
parameter server votes, takes the median and updates.

    python -m paper_2010_04902_b200.worker_step [--steps 30] [--byzantine 3]

The student is one causal layer (attention with a learned relative position bias, a gated feed-forward
block) between an embedding and a vocabulary head, distilled from a fixed teacher's top logits.  Its parameters are one
binary32 vector; a file's gradient is a row of the same length, and bz_glu_backward writes the gated block's weights'
gradients straight into it.  Every one of the r workers that hold a file computes its gradient anew: the vote is exact, so
the step has to give the same bits each time.  The operators of this library do; of the rest only plain products are used
(an embedding's gradient is a product with the tokens' indicator, not a scatter).
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as bz

VOCAB, WIDTH, HEADS, HIDDEN, BUCKETS, DISTANCE = 512, 128, 4, 344, 32, 64
SEQUENCES, LENGTH, TOP = 4, 96, 16

SHAPES = {"embedding": (VOCAB, WIDTH), "wq": (WIDTH, WIDTH), "wk": (WIDTH, WIDTH), "wv": (WIDTH, WIDTH), "wo": (WIDTH, WIDTH),
          "table": (BUCKETS, HEADS), "w_gate": (HIDDEN, WIDTH), "w_up": (HIDDEN, WIDTH), "w_down": (WIDTH, HIDDEN), "head": (VOCAB, WIDTH)}
SIZE = sum(math.prod(s) for s in SHAPES.values())


def views(flat: torch.Tensor) -> dict:
    """The parameters (or their gradients) in a vector of SIZE numbers."""
    out, at = {}, 0
    for name, shape in SHAPES.items():
        n = math.prod(shape)
        out[name] = flat[at:at + n].view(shape)
        at += n
    return out


def initial(seed: int = 0) -> torch.Tensor:
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.zeros(SIZE, device="cuda")
    for name, v in views(w).items():
        if name != "table":
            v.normal_(0.0, 0.3 if name == "embedding" else v.shape[1] ** -0.5, generator=g)
    return w


class Teacher:
    """Top logits that depend on the token and its predecessor, fixed once."""

    def __init__(self, seed: int = 1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        now, before = torch.randn(VOCAB, VOCAB, generator=g, device="cuda"), torch.randn(VOCAB, VOCAB, generator=g, device="cuda")
        self.now, self.before = 2.0 * now, 1.0 * before

    def __call__(self, tokens: torch.Tensor):
        before = torch.cat([tokens[:, :1], tokens[:, :-1]], 1)
        top = (self.now[tokens] + self.before[before]).topk(TOP, dim=-1)
        return top.values.reshape(-1, TOP).contiguous(), top.indices.reshape(-1, TOP).to(torch.int32).contiguous()


def file_gradient(weights: dict, tokens: torch.Tensor, teacher: torch.Tensor, index: torch.Tensor, row: torch.Tensor) -> torch.Tensor:
    """Forward and backward pass of one file; the gradient of the mean loss goes to `row` ([SIZE], binary32).  Returns the
    loss of each position.  `weights`: bfloat16 views (the table binary32)."""
    w, grad = weights, views(row)
    n, t = tokens.shape
    heads = lambda x: x.view(n, t, HEADS, WIDTH // HEADS).transpose(1, 2)  # noqa: E731
    merge = lambda x: x.transpose(1, 2).reshape(n * t, WIDTH)  # noqa: E731
    x = w["embedding"][tokens.reshape(-1)]
    q, k, v = heads(x @ w["wq"].T), heads(x @ w["wk"].T), heads(x @ w["wv"].T)
    scores = q @ k.transpose(2, 3)
    form = {"max_distance": DISTANCE, "bidirectional": False, "causal": True, "scale": (WIDTH // HEADS) ** -0.5}
    probs, stats = bz.bias_softmax(scores, w["table"], **form)
    context = merge(probs @ v)
    y = x + context @ w["wo"].T
    preact = torch.empty(2, n * t, HIDDEN, device="cuda")
    h = bz.glu(y, w["w_gate"], w["w_up"], "gelu_tanh", preact=preact)
    z = y + h @ w["w_down"].T
    logits = z @ w["head"].T
    loss, _, dlogits = bz.distill(logits, teacher, index, 2.0, dloss=torch.full((n * t,), 1.0 / (n * t), device="cuda"))

    grad["head"].copy_(dlogits.T @ z)
    dz = dlogits @ w["head"]
    grad["w_down"].copy_(dz.T @ h)
    dy, _, _ = bz.glu_backward(y, w["w_gate"], w["w_up"], preact, dz @ w["w_down"], "gelu_tanh", dw_gate=grad["w_gate"], dw_up=grad["w_up"])
    dy += dz
    grad["wo"].copy_(dy.T @ context)
    dcontext = heads(dy @ w["wo"])
    dscores, _ = bz.bias_softmax_backward(scores, w["table"], stats, dcontext @ v.transpose(2, 3), dtable=grad["table"], **form)
    dq, dk, dv = merge(dscores @ k), merge(dscores.transpose(2, 3) @ q), merge(probs.transpose(2, 3) @ dcontext)
    dx = dy + dq @ w["wq"] + dk @ w["wk"] + dv @ w["wv"]
    for name, d in (("wq", dq), ("wk", dk), ("wv", dv)):
        grad[name].copy_(d.T @ x)
    indicator = torch.nn.functional.one_hot(tokens.reshape(-1), VOCAB).to(x.dtype)
    grad["embedding"].copy_(indicator.T @ dx)
    return loss


def train(steps: int = 30, byzantine: int = 3, eta: float = 2.0, mu: float = 0.9, seed: int = 0, same_bits: bool = False):
    """Losses of the steps (mean over the files).  `same_bits`: check that every file's honest copies are identical."""
    l, r = 5, 3
    worker_files, file_workers, mask = bz.assign_mols(l, r)
    liars = set()
    if byzantine:
        _, chosen, _ = bz.worst_case(mask, l * l, r, byzantine)
        liars = set(int(j) for j in chosen)
    w, velocity, teacher = initial(seed), torch.zeros(SIZE, device="cuda"), Teacher()
    replicas = torch.empty(r, l * l, SIZE, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    losses = []
    for _ in range(steps):
        half = w.to(torch.bfloat16)
        weights = {**views(half), "table": views(w)["table"]}
        total = 0.0
        for i in range(l * l):
            tokens = torch.randint(0, VOCAB, (SEQUENCES, LENGTH), generator=g, device="cuda")
            top, index = teacher(tokens)
            for k in range(r):   # each worker that holds the file computes it
                loss = file_gradient(weights, tokens, top, index, replicas[k, i])
            total += float(loss.mean())
            if same_bits and not (torch.equal(replicas[0, i], replicas[1, i]) and torch.equal(replicas[0, i], replicas[2, i])):
                raise RuntimeError("two honest copies of file %d differ" % i)
            for k in range(r):
                if int(file_workers[i][k]) in liars:
                    replicas[k, i] *= -100.0   # the reversed-gradient attack
        bz.vote_median_update(replicas, w, eta, velocity, mu)
        losses.append(total / (l * l))
    return losses


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=30)
    p.add_argument("--byzantine", type=int, default=3)
    a = p.parse_args()
    losses = train(a.steps, a.byzantine, same_bits=True)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %3d  loss %.4f" % (i, losses[i]))
    print("step %3d  loss %.4f   (%d parameters, %d of 15 workers reversed their gradients)" % (len(losses) - 1, losses[-1], SIZE, a.byzantine))


if __name__ == "__main__":
    main()
