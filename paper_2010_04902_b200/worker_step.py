"""A small language model trained the ByzShield way: K = 15 workers compute file gradients, some of them lie, the
parameter server votes, takes the median and updates.

    python -m paper_2010_04902_b200.worker_step [--steps 30] [--byzantine 3] [--objective policy|preference] [--dropout 0.1]

The student is one causal layer (attention with a learned relative position bias, a gated feed-forward
block) between an embedding and a vocabulary head, distilled from a fixed teacher's top logits.  Its parameters are one
binary32 vector; a file's gradient is a row of the same length, and bz_glu_backward writes the gated block's weights'
gradients straight into it.  Every one of the r workers that hold a file computes its gradient anew: the vote is exact, so
the step has to give the same bits each time.  The operators of this library do; of the rest only plain products are used
(an embedding's gradient is a product with the tokens' indicator, not a scatter).

With another objective the student is fine-tuned: the clipped policy loss on sampled tokens, or the preference loss on pairs of
sequences.  Its blocks are then joined to the residual stream by bz_join (norms before and behind, gate, dropout), and the attention's
probabilities are dropped by bz_dropout; every worker that holds a file is given the same seed and offset, and so drops
the same elements.
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

# What the joined blocks have besides, kept in binary32.
JOINS = {"norm_in": (WIDTH,), "norm_attention": (WIDTH,), "gate_attention": (1, WIDTH), "norm_block": (WIDTH,), "norm_ffn": (WIDTH,), "gate_ffn": (1, WIDTH),
         "norm_head": (WIDTH,)}
TUNED = {**SHAPES, **JOINS}
TUNED_SIZE = sum(math.prod(s) for s in TUNED.values())


def views(flat: torch.Tensor, shapes: dict = SHAPES) -> dict:
    """The parameters (or their gradients) in a vector of SIZE (or TUNED_SIZE) numbers."""
    out, at = {}, 0
    for name, shape in shapes.items():
        n = math.prod(shape)
        out[name] = flat[at:at + n].view(shape)
        at += n
    return out


def initial(seed: int = 0, shapes: dict = SHAPES) -> torch.Tensor:
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.zeros(sum(math.prod(s) for s in shapes.values()), device="cuda")
    for name, v in views(w, shapes).items():
        if name in JOINS:
            v.fill_(0.5 if name.startswith("gate") else 1.0)
        elif name != "table":
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


def tuned_weights(w: torch.Tensor) -> dict:
    """What tuned_gradient() takes of a parameter vector: bfloat16 matrices, the table and the joins' vectors in binary32."""
    whole = views(w, TUNED)
    return {**views(w.to(torch.bfloat16), TUNED), "table": whole["table"], **{name: whole[name] for name in JOINS}}


def tuned_gradient(weights: dict, tokens: torch.Tensor, objective, rng: torch.Tensor, rate: float, row: torch.Tensor) -> torch.Tensor:
    """file_gradient() of the joined model; the gradient goes to `row` ([TUNED_SIZE], binary32).  objective(logits) gives (losses, their
    gradient in the logits); rng: int64 [3][2], seed and offset of the attention's dropout and of the two joins'."""
    w, grad = weights, views(row, TUNED)
    n, t = tokens.shape
    heads = lambda x: x.view(n, t, HEADS, WIDTH // HEADS).transpose(1, 2)  # noqa: E731
    merge = lambda x: x.transpose(1, 2).reshape(n * t, WIDTH)  # noqa: E731
    form = {"max_distance": DISTANCE, "bidirectional": False, "causal": True, "scale": (WIDTH // HEADS) ** -0.5}
    join1 = {"w_post": w["norm_attention"], "gate": w["gate_attention"], "w_pre": w["norm_block"], "rate": rate, "rng": rng[1]}
    join2 = {"w_post": w["norm_ffn"], "gate": w["gate_ffn"], "w_pre": w["norm_head"], "rate": rate, "rng": rng[2]}
    x = w["embedding"][tokens.reshape(-1)]
    _, a, stats0 = bz.join(x, w_pre=w["norm_in"])
    q, k, v = heads(a @ w["wq"].T), heads(a @ w["wk"].T), heads(a @ w["wv"].T)
    scores = q @ k.transpose(2, 3)
    probs, stats = bz.bias_softmax(scores, w["table"], **form)
    kept = bz.dropout(probs, rate, rng[0])
    context = merge(kept @ v)
    out = context @ w["wo"].T
    s1, y, stats1 = bz.join(x, out, **join1)
    preact = torch.empty(2, n * t, HIDDEN, device="cuda")
    h = bz.glu(y, w["w_gate"], w["w_up"], "gelu_tanh", preact=preact)
    f = h @ w["w_down"].T
    _, z, stats2 = bz.join(s1, f, **join2)
    loss, dlogits = objective(z @ w["head"].T)

    grad["head"].copy_(dlogits.T @ z)
    ds1, df, _, _, _ = bz.join_backward(s1, f, stats2, dz=dlogits @ w["head"], **join2, dw_post=grad["norm_ffn"], dgate=grad["gate_ffn"], dw_pre=grad["norm_head"])
    grad["w_down"].copy_(df.T @ h)
    dy, _, _ = bz.glu_backward(y, w["w_gate"], w["w_up"], preact, df @ w["w_down"], "gelu_tanh", dw_gate=grad["w_gate"], dw_up=grad["w_up"])
    dx, dout, _, _, _ = bz.join_backward(x, out, stats1, ds=ds1, dz=dy, **join1, dw_post=grad["norm_attention"], dgate=grad["gate_attention"], dw_pre=grad["norm_block"])
    grad["wo"].copy_(dout.T @ context)
    dcontext = heads(dout @ w["wo"])
    dprobs = bz.dropout((dcontext @ v.transpose(2, 3)).contiguous(), rate, rng[0])
    dscores, _ = bz.bias_softmax_backward(scores, w["table"], stats, dprobs, dtable=grad["table"], **form)
    dq, dk, dv = merge(dscores @ k), merge(dscores.transpose(2, 3) @ q), merge(kept.transpose(2, 3) @ dcontext)
    for name, d in (("wq", dq), ("wk", dk), ("wv", dv)):
        grad[name].copy_(d.T @ a)
    da = dq @ w["wq"] + dk @ w["wk"] + dv @ w["wv"]
    dx, _, _, _, _ = bz.join_backward(x, None, stats0, ds=dx, dz=da, w_pre=w["norm_in"], dw_pre=grad["norm_in"])
    indicator = torch.nn.functional.one_hot(tokens.reshape(-1), VOCAB).to(x.dtype)
    grad["embedding"].copy_(indicator.T @ dx)
    return loss


def sampled_file(kind: str, teacher: Teacher, g: torch.Generator):
    """One file of a fine-tuning step: (tokens, objective).  Tokens of the teacher's top ones earn an advantage of 1, others -1; a chosen
    sequence is made of the former, the rejected one of the same length of random ones."""
    tokens = torch.randint(0, VOCAB, (SEQUENCES, LENGTH), generator=g, device="cuda")
    _, top = teacher(tokens)
    rows = SEQUENCES * LENGTH
    pick = torch.randint(0, TOP, (rows,), generator=g, device="cuda")
    good = top.gather(1, pick[:, None])[:, 0]
    other = torch.randint(0, VOCAB, (rows,), generator=g, device="cuda", dtype=torch.int32)
    if kind == "policy":
        right = torch.rand(rows, generator=g, device="cuda") < 0.5
        index, advantage = torch.where(right, good, other).contiguous(), torch.where(right, 1.0, -1.0)
        ref = torch.full((rows,), -math.log(VOCAB), device="cuda")
        dloss = torch.full((rows,), 1.0 / rows, device="cuda")

        def objective(logits):
            loss, _, _, dlogits = bz.policy(logits, index, advantage, ref_logp=ref, kl=0.01, dloss=dloss)
            return loss, dlogits
    else:
        pairs = SEQUENCES // 2
        first = torch.arange(rows, device="cuda") < rows // 2
        index = torch.where(first, good, other).contiguous()
        starts = torch.arange(2 * pairs + 1, device="cuda", dtype=torch.int32) * LENGTH
        dloss = torch.full((pairs,), 1.0 / pairs, device="cuda")

        def objective(logits):
            loss, _, _, _, dlogits = bz.preference(logits, index, starts, beta=0.1, mean=True, dloss=dloss)
            return loss, dlogits
    return tokens, objective


def tune(steps: int = 30, byzantine: int = 3, kind: str = "policy", rate: float = 0.1, eta: float = 1.0, mu: float = 0.9, seed: int = 0,
         same_bits: bool = False):
    """train() with the policy or the preference loss on the joined model."""
    l, r = 5, 3
    worker_files, file_workers, mask = bz.assign_mols(l, r)
    liars = set(int(j) for j in bz.worst_case(mask, l * l, r, byzantine)[1]) if byzantine else set()
    w, velocity, teacher = initial(seed, TUNED), torch.zeros(TUNED_SIZE, device="cuda"), Teacher()
    replicas = torch.empty(r, l * l, TUNED_SIZE, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    losses = []
    for step in range(steps):
        weights = tuned_weights(w)
        total = 0.0
        for i in range(l * l):
            tokens, objective = sampled_file(kind, teacher, g)
            rng = torch.tensor([[seed, 3 * (step * l * l + i) + k] for k in range(3)], device="cuda")
            for k in range(r):   # each worker that holds the file computes it
                loss = tuned_gradient(weights, tokens, objective, rng, rate, replicas[k, i])
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
    p.add_argument("--objective", choices=["distill", "policy", "preference"], default="distill")
    p.add_argument("--dropout", type=float, default=0.1, help="of the policy and preference objectives")
    a = p.parse_args()
    if a.objective == "distill":
        losses = train(a.steps, a.byzantine, same_bits=True)
    else:
        losses = tune(a.steps, a.byzantine, a.objective, a.dropout, same_bits=True)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %3d  loss %.4f" % (i, losses[i]))
    print("step %3d  loss %.4f   (%d parameters, %d of 15 workers reversed their gradients)" % (len(losses) - 1, losses[-1], SIZE if a.objective == "distill" else TUNED_SIZE, a.byzantine))


if __name__ == "__main__":
    main()
