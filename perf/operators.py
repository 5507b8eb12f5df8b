"""The operators of a language-model worker's step, as measured cases: a gated feed-forward block, the
softmax of attention scores with a learned relative position bias, and distillation from a teacher's
top logits - each with its gradient.  `own` False: elementary torch operations in 32 bits; `own` True:
the calls of paper_2010_04902_b200.binding.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}
_GELU_C = math.sqrt(2.0 / math.pi)


def listed():
    return [
        # one token through the block: a worker that answers, where latency counts; n = 8/3 of the model width, odd
        {"name": "glu one token", "op": "glu", "part": "forward", "dtype": "f16", "act": "silu", "m": 1, "k": 512, "n": 1365, "pad": 0},
        # a batch of sequences, one token each, weights far larger than the activations
        {"name": "glu 24 tokens", "op": "glu", "part": "forward", "dtype": "bf16", "act": "silu", "m": 24, "k": 2048, "n": 5461, "pad": 0},
        # a file of a few hundred tokens in a small model, ragged in every direction, inputs a slice of a wider buffer
        {"name": "glu train ragged", "op": "glu", "part": "train", "dtype": "f16", "act": "gelu_tanh", "m": 777, "k": 1000, "n": 2666, "pad": 24},
        # a long batch of prompts in a large model, forward only
        {"name": "glu forward large", "op": "glu", "part": "forward", "dtype": "bf16", "act": "silu", "m": 8192, "k": 4096, "n": 10922, "pad": 0},
        # one file of a large model's training step: forward, then all three gradients
        {"name": "glu train large", "op": "glu", "part": "train", "dtype": "bf16", "act": "gelu_tanh", "m": 8192, "k": 4096, "n": 8192, "pad": 0},
        # one step of a generated sequence: a single query against ragged caches
        {"name": "bias one query", "op": "bias", "part": "forward", "dtype": "bf16", "b": 16, "h": 16, "tq": 1, "tk": 8192, "buckets": 32,
         "distance": 128, "both": False, "causal": False, "ragged": True, "pad": 0},
        # a long prompt, causal
        {"name": "bias prompt causal", "op": "bias", "part": "forward", "dtype": "bf16", "b": 2, "h": 16, "tq": 4096, "tk": 4096, "buckets": 32,
         "distance": 128, "both": False, "causal": True, "ragged": False, "pad": 0},
        # a small encoder-decoder file in 32 bits: odd lengths, padded rows, keys of different lengths
        {"name": "bias train ragged", "op": "bias", "part": "train", "dtype": "f32", "b": 3, "h": 6, "tq": 333, "tk": 517, "buckets": 32,
         "distance": 128, "both": True, "causal": False, "ragged": True, "pad": 3},
        # an encoder layer's training step
        {"name": "bias train", "op": "bias", "part": "train", "dtype": "bf16", "b": 8, "h": 16, "tq": 1024, "tk": 1024, "buckets": 32,
         "distance": 128, "both": True, "causal": False, "ragged": False, "pad": 0},
        # a handful of positions in 32 bits, loss and gradient in one call
        {"name": "distill small", "op": "distill", "part": "train", "dtype": "f32", "m": 32, "v": 10007, "t": 16, "temperature": 2.0, "pad": 0},
        # scoring a held-out batch: the loss alone, a large odd vocabulary
        {"name": "distill loss", "op": "distill", "part": "forward", "dtype": "f16", "m": 2048, "v": 100003, "t": 50, "temperature": 1.0, "pad": 5},
        # one file of a training step
        {"name": "distill train", "op": "distill", "part": "train", "dtype": "bf16", "m": 4096, "v": 32128, "t": 64, "temperature": 2.0, "pad": 0},
    ]


def _spread(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; half of them multiples of 8 where that is possible."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 16 and rng.random() < 0.5:
        n = n // 8 * 8
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(["glu", "bias", "distill"])
    if op == "glu":
        while True:
            c = {"op": op, "part": rng.choice(["forward", "train"]), "dtype": rng.choice(["bf16", "f16"]),
                 "act": rng.choice(["silu", "gelu_tanh"]), "m": _spread(rng, 1, 8192), "k": _spread(rng, 64, 4096),
                 "n": _spread(rng, 64, 10922), "pad": rng.choice([0, 0, 8, 13])}
            if work(c)["flops"] <= 12 * 8192 * 4096 * 8192:
                return c
    if op == "bias":
        while True:
            part = rng.choice(["forward", "train", "query"])
            both = rng.random() < 0.5
            c = {"op": op, "part": "train" if part == "train" else "forward", "dtype": rng.choice(["bf16", "f16", "f32"]),
                 "b": rng.randint(1, 16), "h": rng.randint(1, 32), "tq": 1 if part == "query" else _spread(rng, 2, 4096), "tk": _spread(rng, 1, 8192),
                 "buckets": rng.choice([16, 32, 64]), "distance": rng.choice([64, 128, 200]), "both": both,
                 "causal": not both and part != "query", "ragged": rng.random() < 0.5, "pad": rng.choice([0, 0, 3, 8])}
            if c["b"] * c["h"] * c["tq"] * c["tk"] <= 8 * 16 * 1024 * 1024:
                return c
    while True:
        c = {"op": op, "part": rng.choice(["forward", "train"]), "dtype": rng.choice(["bf16", "f16", "f32"]), "m": _spread(rng, 1, 8192),
             "v": _spread(rng, 500, 200000), "t": _spread(rng, 1, 128), "temperature": rng.choice([1.0, 2.0, 4.0]), "pad": rng.choice([0, 0, 5, 8])}
        if c["m"] * c["v"] <= 4096 * 32128:
            return c


# ---- inputs ---------------------------------------------------------------------------------------


def _wide(shape, pad, dtype, gen, sigma=1.0):
    """Normal values in a tensor whose last dimension is a slice of one `pad` elements longer."""
    full = torch.empty(*shape[:-1], shape[-1] + pad, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=gen)
    return full[..., : shape[-1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "glu":
        # normalised activations, weights of the usual initial scale, a loss-scaled gradient of order one
        m, k, n = case["m"], case["k"], case["n"]
        s["x"] = _wide((m, k), case["pad"], dt, gen)
        s["w_gate"] = _wide((n, k), 0, dt, gen, k ** -0.5)
        s["w_up"] = _wide((n, k), 0, dt, gen, k ** -0.5)
        if case["part"] == "train":
            s["dh"] = _wide((m, n), 0, dt, gen)
    elif case["op"] == "bias":
        b, h, tq, tk = case["b"], case["h"], case["tq"], case["tk"]
        s["scores"] = _wide((b, h, tq, tk), case["pad"], dt, gen, 2.0)
        s["table"] = torch.empty(case["buckets"], h, device="cuda").normal_(0.0, 1.0, generator=gen)
        s["k_len"] = torch.randint(1, tk + 1, (b,), generator=gen, device="cuda", dtype=torch.int32) if case["ragged"] else None
        # a single query stands at the end of its keys; otherwise the queries begin where the keys do
        if tq == 1:
            s["q_start"] = (s["k_len"] - 1) if case["ragged"] else torch.full((b,), tk - 1, dtype=torch.int32, device="cuda")
        else:
            s["q_start"] = None
        if case["part"] == "train":
            s["dprobs"] = _wide((b, h, tq, tk), 0, dt, gen)
    else:
        m, v, t = case["m"], case["v"], case["t"]
        s["logits"] = _wide((m, v), case["pad"], dt, gen, 2.5)
        # the teacher's largest logits lie where the student's tend to be large too; a twentieth of the positions is padding
        # and has no teacher, a tenth has half of the entries only
        top = (s["logits"].float() + torch.empty(m, v, device="cuda").normal_(0.0, 2.0, generator=gen)).topk(t, dim=1)
        s["teacher"] = top.values.contiguous()
        index = top.indices.to(torch.int32)
        u = torch.rand(m, 1, generator=gen, device="cuda")
        col = torch.arange(t, device="cuda")[None, :]
        gone = (u < 0.05) | ((u < 0.15) & (col >= (t + 1) // 2))
        s["index"] = torch.where(gone, torch.full_like(index, -1), index).contiguous()
        if case["part"] == "train":
            s["dloss"] = torch.empty(m, device="cuda").uniform_(0.5, 1.5, generator=gen)
    return s


# ---- plain forms ----------------------------------------------------------------------------------


def _act(name, g):
    """The activation and its derivative."""
    if name == "silu":
        e = 1.0 / (1.0 + torch.exp(-g))
        return g * e, e * (1.0 + g * (1.0 - e))
    u = _GELU_C * (g + 0.044715 * g * g * g)
    t = torch.tanh(u)
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * _GELU_C * (1.0 + 3 * 0.044715 * g * g)


def _plain_glu(s):
    c = s["case"]
    dt = s["x"].dtype
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    g, u = x @ wg.T, x @ wu.T
    a, da = _act(c["act"], g)
    out = {"h": (a * u).to(dt)}
    if c["part"] == "train":
        dh = s["dh"].float()
        dg, du = dh * u * da, dh * a
        out["dx"] = (dg @ wg + du @ wu).to(dt)
        out["dw_gate"] = (dg.T @ x).to(dt)
        out["dw_up"] = (du.T @ x).to(dt)
    return out


def _starts(buckets, distance):
    """The distances at which the buckets beyond the exact half begin."""
    exact = buckets // 2
    steps = buckets - exact
    n, got = exact, []
    for j in range(1, steps):
        while n ** steps < exact ** (steps - j) * distance ** j:
            n += 1
        got.append(n)
    return exact, got


def _bucket_of(case, rel):
    """The bucket of each relative position (key minus query)."""
    nb = case["buckets"] // 2 if case["both"] else case["buckets"]
    exact, starts = _starts(nb, case["distance"])
    near = torch.arange(case["distance"] + 1, device=rel.device)
    lut = near.clamp(max=exact) + (near[:, None] >= torch.tensor(starts, device=rel.device, dtype=torch.long)[None, :]).sum(1)
    if case["both"]:
        return lut[rel.abs().clamp(max=case["distance"])] + nb * (rel > 0)
    return lut[(-rel).clamp(min=0, max=case["distance"])]


def _positions(s):
    """(rel, visible), each [b or 1, tq, tk]."""
    c = s["case"]
    i = torch.arange(c["tq"], device="cuda")[None, :, None]
    j = torch.arange(c["tk"], device="cuda")[None, None, :]
    q = i if s["q_start"] is None else i + s["q_start"].long()[:, None, None]
    rel = j - q
    seen = torch.ones_like(rel, dtype=torch.bool)
    if c["causal"]:
        seen = rel <= 0
    if s["k_len"] is not None:
        seen = seen & (j < s["k_len"].long()[:, None, None])
    return rel, seen


def _plain_bias(s):
    c = s["case"]
    dt = s["scores"].dtype
    rel, seen = _positions(s)
    bucket = _bucket_of(c, rel)
    z = s["scores"].float() + s["table"][bucket].permute(0, 3, 1, 2)
    z = torch.where(seen[:, None], z, torch.full_like(z, -math.inf))
    top = z.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, torch.zeros_like(e))
    out = {"probs": p.to(dt)}
    if c["part"] == "train":
        dp = s["dprobs"].float()
        dz = p * (dp - (p * dp).sum(-1, keepdim=True))
        out["dscores"] = dz.to(dt)
        # rows first, then their sum: a single chain of additions over all positions would lose the last digits
        d = dz.sum(0, keepdim=True) if bucket.shape[0] == 1 else dz
        hot = (bucket[..., None] == torch.arange(c["buckets"], device="cuda")).float()
        out["dtable"] = (d.permute(0, 2, 1, 3) @ hot).sum((0, 1)).T.contiguous()
    return out


def _plain_distill(s):
    c = s["case"]
    T = c["temperature"]
    there = s["index"] >= 0
    any_there = there.any(1)
    at = s["index"].long().clamp(min=0)
    t = torch.where(there, s["teacher"] / T, torch.full_like(s["teacher"], -math.inf))
    t = torch.where(any_there[:, None], t - t.amax(1, keepdim=True), t)
    e = torch.where(there, torch.exp(t), torch.zeros_like(t))
    total = torch.where(any_there, e.sum(1), torch.ones_like(any_there, dtype=torch.float32))
    p = e / total[:, None]
    z = s["logits"].float() / T
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    norm = e.sum(1, keepdim=True)
    log_q = z.gather(1, at) - top - torch.log(norm)
    log_p = t - torch.log(total)[:, None]
    loss = T * T * torch.where(there, p * (log_p - log_q), torch.zeros_like(p)).sum(1)
    out = {"loss": loss}
    if c["part"] == "train":
        d = torch.where(any_there[:, None], e / norm, torch.zeros_like(e)).scatter_add(1, at, -p)
        out["dlogits"] = (s["dloss"][:, None] * T * d).to(s["logits"].dtype)
    return out


# ---- one pass -------------------------------------------------------------------------------------


def run(state):
    c = state["case"]
    if not own:
        return {"glu": _plain_glu, "bias": _plain_bias, "distill": _plain_distill}[c["op"]](state)
    from paper_2010_04902_b200 import binding as bz
    if c["op"] == "glu":
        x, wg, wu = state["x"], state["w_gate"], state["w_up"]
        if c["part"] == "forward":
            return {"h": bz.glu(x, wg, wu, c["act"])}
        preact = torch.empty(2, c["m"], c["n"], dtype=torch.float32, device="cuda")
        h = bz.glu(x, wg, wu, c["act"], preact=preact)
        dx, dwg, dwu = bz.glu_backward(x, wg, wu, preact, state["dh"], c["act"])
        return {"h": h, "dx": dx, "dw_gate": dwg, "dw_up": dwu}
    if c["op"] == "bias":
        form = {"max_distance": c["distance"], "bidirectional": c["both"], "causal": c["causal"], "k_len": state["k_len"], "q_start": state["q_start"]}
        probs, lse = bz.bias_softmax(state["scores"], state["table"], **form)
        if c["part"] == "forward":
            return {"probs": probs}
        dscores, dtable = bz.bias_softmax_backward(state["scores"], state["table"], lse, state["dprobs"], **form)
        return {"probs": probs, "dscores": dscores, "dtable": dtable}
    if c["part"] == "forward":
        loss, _ = bz.distill(state["logits"], state["teacher"], state["index"], c["temperature"])
        return {"loss": loss}
    loss, _, dlogits = bz.distill(state["logits"], state["teacher"], state["index"], c["temperature"], dloss=state["dloss"])
    return {"loss": loss, "dlogits": dlogits}


def work(case):
    e = _SIZE[case["dtype"]]
    train = case["part"] == "train"
    if case["op"] == "glu":
        m, k, n = case["m"], case["k"], case["n"]
        # x, both weights and h; then dh, dx and both weights' gradients
        bytes_ = e * (m * k + 2 * n * k + m * n)
        if train:
            bytes_ += e * (m * n + m * k + 2 * n * k)
        return {"bytes": bytes_, "flops": (12 if train else 4) * m * n * k}
    if case["op"] == "bias":
        size = case["b"] * case["h"] * case["tq"] * case["tk"]
        # scores and probabilities, then their gradients; four operations an element forward, six backward
        return {"bytes": e * size * (4 if train else 2) + 4 * case["buckets"] * case["h"] * (2 if train else 1), "flops": (10 if train else 4) * size}
    size = case["m"] * case["v"]
    return {"bytes": e * size * (2 if train else 1) + case["m"] * (8 * case["t"] + 4 + (4 if train else 0)), "flops": (6 if train else 3) * size}


# ---- the definition in 64 bits --------------------------------------------------------------------


def _exact_glu(case, s):
    x, a, b = (s[k].double() for k in ("x", "w_gate", "w_up"))
    g, u = torch.einsum("mk,nk->mn", x, a), torch.einsum("mk,nk->mn", x, b)
    if case["act"] == "silu":
        sig = torch.sigmoid(g)
        f, df = g * sig, sig + g * sig * torch.sigmoid(-g)
    else:
        # 0.5 (1 + tanh y) = sigmoid(2 y)
        sig = torch.sigmoid(2 * _GELU_C * (g + 0.044715 * g ** 3))
        f, df = g * sig, sig + g * sig * (1 - sig) * 2 * _GELU_C * (1 + 0.134145 * g ** 2)
    out = {"h": f * u}
    if case["part"] == "train":
        dh = s["dh"].double()
        f *= dh
        df *= dh * u
        out["dx"] = torch.einsum("mn,nk->mk", df, a) + torch.einsum("mn,nk->mk", f, b)
        out["dw_gate"] = torch.einsum("mn,mk->nk", df, x)
        out["dw_up"] = torch.einsum("mn,mk->nk", f, x)
    return out


def _exact_bias(case, s):
    b, h, tq, tk = case["b"], case["h"], case["tq"], case["tk"]
    nb = case["buckets"] // 2 if case["both"] else case["buckets"]
    exact, starts = _starts(nb, case["distance"])

    def bucket(rel):
        far = 0
        if case["both"] and rel > 0:
            far = nb
        n = abs(rel) if case["both"] else max(-rel, 0)
        return far + (n if n < exact else exact + sum(n >= at for at in starts))

    probs = torch.zeros(b, h, tq, tk, dtype=torch.float64, device="cuda")
    dscores = torch.zeros_like(probs) if case["part"] == "train" else None
    dtable = torch.zeros(case["buckets"], h, dtype=torch.float64, device="cuda")
    for n in range(b):
        start = int(s["q_start"][n]) if s["q_start"] is not None else 0
        keys = int(s["k_len"][n]) if s["k_len"] is not None else tk
        # every relative position from the last query's first key to the first query's last key
        by_rel = torch.tensor([bucket(r) for r in range(-(start + tq - 1), tk - start)], device="cuda")
        at = torch.arange(keys, device="cuda")[None, :] - torch.arange(tq, device="cuda")[:, None] + tq - 1
        kind = by_rel[at]
        z = s["scores"][n, :, :, :keys].double() + s["table"].double().T[:, kind]
        if case["causal"]:
            z.masked_fill_(at > start + tq - 1, -math.inf)
        p = torch.softmax(z, -1)
        probs[n, :, :, :keys] = p
        if dscores is not None:
            dp = s["dprobs"][n, :, :, :keys].double()
            dz = p * dp
            dz -= p * dz.sum(-1, keepdim=True)
            dscores[n, :, :, :keys] = dz
            dtable.index_add_(0, kind.reshape(-1), dz.reshape(h, -1).T)
    return {"probs": probs, "dscores": dscores, "dtable": dtable} if dscores is not None else {"probs": probs}


def _exact_distill(case, s):
    T, m, t = case["temperature"], case["m"], case["t"]
    logits = s["logits"].double() / T
    log_q = logits - torch.logsumexp(logits, 1, keepdim=True)
    there = s["index"] >= 0
    full = torch.where(there, s["teacher"].double() / T, torch.full((m, t), -math.inf, dtype=torch.float64, device="cuda"))
    log_p = full - torch.logsumexp(full, 1, keepdim=True)
    log_p = torch.where(there, log_p, torch.zeros_like(log_p))
    p = torch.where(there, torch.exp(log_p), torch.zeros_like(log_p))
    row, col = torch.nonzero(there, as_tuple=True)
    cell = s["index"].long()[row, col]
    loss = torch.zeros(m, dtype=torch.float64, device="cuda")
    loss.index_add_(0, row, p[row, col] * (log_p[row, col] - log_q[row, cell]))
    out = {"loss": T * T * loss}
    if case["part"] == "train":
        d = torch.exp(log_q) * p.sum(1, keepdim=True)
        d.index_put_((row, cell), -p[row, col], accumulate=True)
        out["dlogits"] = s["dloss"].double()[:, None] * T * d
    return out


def exact(case, seed):
    return {"glu": _exact_glu, "bias": _exact_bias, "distill": _exact_distill}[case["op"]](case, prepare(case, seed))
