"""More operators of a language-model worker's step, as measured cases: the clipped policy loss with a KL term and the
paired preference loss (beside distillation), the join of a block to its residual stream (norm after the block, gate,
dropout, residual scale, norm before the next block) and dropout from a counter-based generator - each with its
gradient.  `own` False: elementary torch operations; `own` True: the calls of paper_2010_04902_b200.binding.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}
_CELLS = 4096 * 32128        # logits of the largest loss case
_ELEMENTS = 8192 * 16384     # elements of the largest join and dropout cases


def listed():
    return [
        # a handful of positions in 32 bits, loss and gradient in one call
        {"name": "policy few positions", "op": "policy", "part": "train", "dtype": "f32", "m": 24, "v": 10007, "temperature": 1.0, "kl": 0.05, "pad": 0},
        # scoring what was generated: loss and log-probabilities alone, odd vocabulary, rows of a wider buffer
        {"name": "policy loss", "op": "policy", "part": "forward", "dtype": "f16", "m": 1531, "v": 65537, "temperature": 0.7, "kl": 0.05, "pad": 5},
        # one file of a training step
        {"name": "policy train", "op": "policy", "part": "train", "dtype": "bf16", "m": 4096, "v": 32128, "temperature": 1.0, "kl": 0.02, "pad": 0},
        # a file of a model with a large vocabulary, no KL term
        {"name": "policy train wide", "op": "policy", "part": "train", "dtype": "bf16", "m": 1024, "v": 128000, "temperature": 1.0, "kl": 0.0, "pad": 0},
        # three short ragged pairs in 32 bits
        {"name": "preference ragged", "op": "preference", "part": "train", "dtype": "f32", "m": 187, "v": 5003, "pairs": 3, "mean": False,
         "smoothing": 0.1, "pad": 3},
        # one file of a training step: eight pairs of answers of some hundred tokens
        {"name": "preference train", "op": "preference", "part": "train", "dtype": "bf16", "m": 4096, "v": 32128, "pairs": 8, "mean": False,
         "smoothing": 0.0, "pad": 0},
        # one token between two blocks of a model that answers, where latency counts
        {"name": "join one token", "op": "join", "part": "forward", "dtype": "bf16", "m": 1, "n": 4096, "norm": "rms", "post": True, "groups": 1,
         "residual": 1.0, "branch": 1.0, "rate": 0.0, "pad": 0},
        # a long batch of prompts through a wide model, a gate for each sequence, no norm behind the block
        {"name": "join forward wide", "op": "join", "part": "forward", "dtype": "f16", "m": 16384, "n": 8192, "norm": "rms", "post": False, "groups": 16,
         "residual": 1.0, "branch": 0.5, "rate": 0.0, "pad": 0},
        # a file of a small model in 32 bits: layer norms, odd sizes, padded rows
        {"name": "join train ragged", "op": "join", "part": "train", "dtype": "f32", "m": 777, "n": 1001, "norm": "layer", "post": True, "groups": 3,
         "residual": 1.7, "branch": 1.0, "rate": 0.1, "pad": 3},
        # one file of a large model's training step
        {"name": "join train", "op": "join", "part": "train", "dtype": "bf16", "m": 8192, "n": 4096, "norm": "rms", "post": True, "groups": 1,
         "residual": 1.0, "branch": 1.0, "rate": 0.1, "pad": 0},
        # a small encoder-decoder file's attention probabilities in 32 bits, rows of a wider buffer
        {"name": "dropout ragged", "op": "dropout", "part": "train", "dtype": "f32", "m": 5994, "n": 517, "rate": 0.1, "pad": 3},
        # the attention probabilities of an encoder layer's training step
        {"name": "dropout train", "op": "dropout", "part": "train", "dtype": "bf16", "m": 8 * 16 * 1024, "n": 1024, "rate": 0.1, "pad": 0},
    ]


def _spread(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; half of them multiples of 8 where that is possible."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 16 and rng.random() < 0.5:
        n = n // 8 * 8
    return max(lo, min(hi, n))


def draw(rng):
    op = rng.choice(["policy", "preference", "join", "dropout"])
    common = {"op": op, "part": rng.choice(["forward", "train"]), "dtype": rng.choice(["bf16", "f16", "f32"]), "pad": rng.choice([0, 0, 5, 8])}
    while True:
        if op == "policy":
            c = {"m": _spread(rng, 1, 8192), "v": _spread(rng, 500, 200000), "temperature": rng.choice([0.7, 1.0, 1.5]), "kl": rng.choice([0.0, 0.02, 0.1])}
            if c["m"] * c["v"] <= _CELLS // 2:
                return {**common, **c}
        elif op == "preference":
            c = {"m": _spread(rng, 8, 8192), "v": _spread(rng, 500, 200000), "pairs": rng.randint(1, 16), "mean": rng.random() < 0.3,
                 "smoothing": rng.choice([0.0, 0.1])}
            if c["m"] * c["v"] <= _CELLS // 2 and c["pairs"] * 4 <= c["m"]:
                return {**common, **c}
        elif op == "join":
            groups = rng.choice([0, 1, 1, 4, 7])
            c = {"m": _spread(rng, 1, 16384), "n": _spread(rng, 64, 16384), "norm": rng.choice(["rms", "rms", "layer"]), "post": rng.random() < 0.6,
                 "groups": groups, "residual": rng.choice([1.0, 1.0, 1.7]), "branch": rng.choice([1.0, 0.5]), "rate": rng.choice([0.0, 0.1, 0.25])}
            c["m"] = max(groups, c["m"] // max(1, groups) * max(1, groups))
            if c["m"] * c["n"] <= 8192 * 4096:
                return {**common, **c}
        else:
            c = {"m": _spread(rng, 1, 1 << 20), "n": _spread(rng, 1, 16384), "rate": rng.choice([0.1, 0.1, 0.25, 0.5])}
            if 4096 <= c["m"] * c["n"] <= _ELEMENTS:
                return {**common, **c}


# ---- inputs ---------------------------------------------------------------------------------------


def _wide(shape, pad, dtype, gen, sigma=1.0):
    """Normal values in a tensor whose last dimension is a slice of one `pad` elements longer."""
    full = torch.empty(*shape[:-1], shape[-1] + pad, dtype=dtype, device="cuda").normal_(0.0, sigma, generator=gen)
    return full[..., : shape[-1]]


def _normal(shape, gen, sigma=1.0, mean=0.0):
    return torch.empty(shape, device="cuda").normal_(mean, sigma, generator=gen)


def _sampled(logits, temperature, gen):
    """Tokens drawn from softmax(logits / T), and their log-probabilities in 64 bits; a slice of the rows at a time."""
    m, v = logits.shape
    index, logp = torch.empty(m, dtype=torch.int32, device="cuda"), torch.empty(m, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 25) // v)
    for a in range(0, m, step):
        z = logits[a:a + step].float() / temperature
        # the largest of z + a Gumbel variable is a draw from softmax(z)
        noise = torch.empty_like(z).exponential_(generator=gen)
        at = (z - torch.log(noise)).argmax(1)
        index[a:a + step] = at.to(torch.int32)
        z = logits[a:a + step].double() / temperature
        logp[a:a + step] = z.gather(1, at[:, None])[:, 0] - torch.logsumexp(z, 1)
    return index, logp


_CLIP_LOW, _CLIP_HIGH, _BETA, _MARGIN = 0.2, 0.28, 0.1, 0.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _DTYPES[case["dtype"]]
    op, train = case["op"], case["part"] == "train"
    s = {"case": case}
    if op in ("policy", "preference"):
        m, v = case["m"], case["v"]
        s["logits"] = _wide((m, v), case["pad"], dt, gen, 2.5)
        s["index"], logp = _sampled(s["logits"], case.get("temperature", 1.0), gen)
        # a twentieth of the positions is a prompt's or padding: no token was chosen there
        s["index"][torch.rand(m, generator=gen, device="cuda") < 0.05] = -1
        # the reference is an earlier model: near, not equal
        s["ref"] = (logp + _normal(m, gen, 0.2).double()).float()
        if op == "policy":
            # the policy that generated is some steps old.  The gradient jumps where the ratio meets a border of the clip; a
            # ratio within rounding of it may fall on either side, so none is left there
            moved = _normal(m, gen, 0.2)
            for border in (math.log(1 - _CLIP_LOW), math.log(1 + _CLIP_HIGH)):
                moved = torch.where((moved - border).abs() < 1e-3, moved + 4e-3, moved)
            s["old"] = (logp - moved.double()).float()
            s["advantage"] = _normal(m, gen)
            s["dloss"] = torch.empty(m, device="cuda").uniform_(0.5, 1.5, generator=gen)
        else:
            # sequences of different lengths, chosen ones first; some rows behind the last sequence are nobody's
            n = 2 * case["pairs"]
            used = max(n, m - m // 50)
            weight = torch.rand(n, generator=gen, device="cuda") + 0.3
            ends = (weight.cumsum(0) / weight.sum() * used).round().to(torch.int32)
            s["starts"] = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), ends])
            s["dloss"] = torch.empty(case["pairs"], device="cuda").uniform_(0.5, 1.5, generator=gen)
    elif op == "join":
        m, n = case["m"], case["n"]
        s["x"] = _wide((m, n), case["pad"], dt, gen, 2.0)
        s["y"] = _wide((m, n), case["pad"], dt, gen, 0.7)
        s["w_post"] = _normal(n, gen, 0.1, 1.0) if case["post"] else None
        s["w_pre"] = _normal(n, gen, 0.1, 1.0)
        s["gate"] = _normal((case["groups"], n), gen, 0.3, 0.5) if case["groups"] else None
        s["rng"] = torch.randint(0, 1 << 62, (2,), generator=gen, device="cuda") if case["rate"] else None
        if train:
            s["ds"], s["dz"] = _wide((m, n), 0, dt, gen), _wide((m, n), 0, dt, gen)
    else:
        m, n = case["m"], case["n"]
        s["x"] = _wide((m, n), case["pad"], dt, gen)
        s["rng"] = torch.randint(0, 1 << 62, (2,), generator=gen, device="cuda")
        if train:
            s["dout"] = _wide((m, n), 0, dt, gen)
    return s


# ---- plain forms ----------------------------------------------------------------------------------


def _plain_logp(logits, index, temperature):
    """(exponentials of the row, their sum, log-probability of the row's token, whether it has one)."""
    z = logits.float() / temperature
    z = z - z.amax(1, keepdim=True)
    there = (index >= 0) & (index < logits.shape[1])
    at = torch.where(there, index, torch.zeros_like(index)).long()[:, None]
    chosen = z.gather(1, at)[:, 0].double()
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    logp = torch.where(there, chosen - torch.log(total[:, 0].double()), torch.zeros_like(chosen))
    return e, total, logp, there, at


def _plain_dlogits(e, total, there, at, g, dtype):
    """g * (indicator of the token - softmax)."""
    g = torch.where(there, g, torch.zeros_like(g))[:, None]
    return (e * (-g / total)).scatter_add(1, at, g).to(dtype)


def _plain_policy(s):
    c = s["case"]
    e, total, logp, there, at = _plain_logp(s["logits"], s["index"], c["temperature"])
    # row scalars in 64 bits: next to a border of the clip, and where exp(d) - d - 1 is small, 32 would lose what matters
    adv = s["advantage"].double()
    ratio = torch.exp(logp - s["old"].double())
    clipped = torch.minimum(torch.maximum(ratio, torch.full_like(ratio, 1 - _CLIP_LOW)), torch.full_like(ratio, 1 + _CLIP_HIGH))
    d = s["ref"].double() - logp
    loss = -torch.minimum(ratio * adv, clipped * adv) + c["kl"] * (torch.exp(d) - d - 1)
    zero = torch.zeros_like(loss)
    out = {"loss": torch.where(there, loss, zero).float(), "logp": logp.float()}
    if c["part"] == "train":
        held = ((adv > 0) & (ratio > 1 + _CLIP_HIGH)) | ((adv < 0) & (ratio < 1 - _CLIP_LOW))
        g = torch.where(held, zero, -ratio * adv) + c["kl"] * (1 - torch.exp(d))
        out["dlogits"] = _plain_dlogits(e, total, there, at, (g * s["dloss"] / c["temperature"]).float(), s["logits"].dtype)
    return out


def _plain_preference(s):
    c = s["case"]
    m, pairs = c["m"], c["pairs"]
    e, total, logp, there, at = _plain_logp(s["logits"], s["index"], 1.0)
    starts = s["starts"].long()
    row = torch.arange(m, device="cuda")
    member = (row[None, :] >= starts[:-1, None]) & (row[None, :] < starts[1:, None]) & there[None, :]
    apart = torch.where(there, logp - s["ref"].double(), torch.zeros_like(logp))
    share = member.double()
    if c["mean"]:
        share = share / share.sum(1, keepdim=True).clamp(min=1.0)
    reward = _BETA * (share * apart[None, :]).sum(1)
    h = reward[:pairs] - reward[pairs:] - _MARGIN
    eps = c["smoothing"]
    # log sigmoid(h) = min(h, 0) - log(1 + exp(-|h|))
    tail = torch.log(1 + torch.exp(-h.abs()))
    loss = -(1 - eps) * (h.clamp(max=0.0) - tail) - eps * ((-h).clamp(max=0.0) - tail)
    out = {"loss": loss.float(), "reward": reward.float(), "logp": logp.float()}
    if c["part"] == "train":
        dh = 1 / (1 + torch.exp(-h)) - (1 - eps)
        dreward = torch.cat([dh * s["dloss"], -dh * s["dloss"]]) * _BETA
        g = (share * dreward[:, None]).sum(0).float()
        out["dlogits"] = _plain_dlogits(e, total, there, at, g, s["logits"].dtype)
    return out


def _low(x):
    return x & 0xFFFFFFFF


def _mul32(a, b):
    """High and low 32 bits of a * b for 0 <= a < 2^32 in an int64 tensor and a constant b < 2^32."""
    lo, hi = a * (b & 0xFFFF), a * (b >> 16)        # below 2^48 each
    mid = hi + (lo >> 16)
    return mid >> 16, _low((mid << 16) | (lo & 0xFFFF))


def _plain_kept(rng, m, n, rate):
    """Which elements of an [m][n] tensor stay: those whose 16 random bits are at least round(65536 rate).  Eight elements in
    row-major order share one output of Philox4x32-10 (Salmon et al., 2011): counter (their number / 8, offset), key seed."""
    count = (m * n + 7) // 8
    number = torch.arange(count, device="cuda")
    x = [_low(number), number >> 32, _low(rng[1]).expand(count), _low(rng[1] >> 32).expand(count)]
    k0, k1 = _low(rng[0]), _low(rng[0] >> 32)
    for _ in range(10):
        h0, l0 = _mul32(x[0], 0xD2511F53)
        h1, l1 = _mul32(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
        k0, k1 = _low(k0 + 0x9E3779B9), _low(k1 + 0xBB67AE85)
    bits = torch.stack([h for w in x for h in (w & 0xFFFF, w >> 16)], 1)
    return (bits >= int(round(rate * 65536))).reshape(-1)[: m * n].view(m, n)


def _drop_scale(rate):
    return 65536.0 / (65536.0 - round(rate * 65536))


def _plain_norm(x, w, kind, eps=1e-6):
    """(norm of x's rows times w, normalised rows, 1 / deviation)."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    r = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
    return x * r * w, x * r, r


def _plain_norm_backward(dz, w, hat, r, kind):
    """(gradient of the norm's input, of its weight)."""
    d = dz * w
    dx = d - hat * (d * hat).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - d.mean(1, keepdim=True)
    return dx * r, (dz * hat).sum(0)


def _plain_join(s):
    c = s["case"]
    m, n, kind = c["m"], c["n"], c["norm"]
    dt = s["x"].dtype
    x, y = s["x"].float(), s["y"].float()
    a = y
    if c["post"]:
        a, y_hat, y_r = _plain_norm(y, s["w_post"], kind)
    gate = s["gate"].repeat_interleave(m // c["groups"], 0) if c["groups"] else torch.ones(1, n, device="cuda")
    factor = torch.full((1, 1), c["branch"], device="cuda")
    if c["rate"]:
        factor = torch.where(_plain_kept(s["rng"], m, n, c["rate"]), factor * _drop_scale(c["rate"]), torch.zeros_like(factor))
    t = c["residual"] * x + factor * gate * a
    z, hat, r = _plain_norm(t, s["w_pre"], kind)
    out = {"s": t.to(dt), "z": z.to(dt)}
    if c["part"] == "train":
        dt_, out["dw_pre"] = _plain_norm_backward(s["dz"].float(), s["w_pre"], hat, r, kind)
        dt_ = dt_ + s["ds"].float()
        out["dx"] = (c["residual"] * dt_).to(dt)
        if c["groups"]:
            out["dgate"] = (factor * a * dt_).view(c["groups"], m // c["groups"], n).sum(1)
        da = factor * gate * dt_
        if c["post"]:
            da, out["dw_post"] = _plain_norm_backward(da, s["w_post"], y_hat, y_r, kind)
        out["dy"] = da.to(dt)
    return out


def _plain_dropout(s):
    c = s["case"]
    kept = _plain_kept(s["rng"], c["m"], c["n"], c["rate"])
    zero = torch.zeros((), device="cuda")
    out = {"out": torch.where(kept, s["x"].float() * _drop_scale(c["rate"]), zero).to(s["x"].dtype)}
    if c["part"] == "train":
        out["dx"] = torch.where(kept, s["dout"].float() * _drop_scale(c["rate"]), zero).to(s["x"].dtype)
    return out


# ---- one pass -------------------------------------------------------------------------------------


def run(state):
    c = state["case"]
    if not own:
        return {"policy": _plain_policy, "preference": _plain_preference, "join": _plain_join, "dropout": _plain_dropout}[c["op"]](state)
    from paper_2010_04902_b200 import binding as bz
    train = c["part"] == "train"
    if c["op"] == "policy":
        got = bz.policy(state["logits"], state["index"], state["advantage"], old_logp=state["old"], ref_logp=state["ref"], kl=c["kl"],
                        clip_low=_CLIP_LOW, clip_high=_CLIP_HIGH, temperature=c["temperature"], dloss=state["dloss"] if train else None)
        out = {"loss": got[0], "logp": got[1]}
    elif c["op"] == "preference":
        got = bz.preference(state["logits"], state["index"], state["starts"], ref_logp=state["ref"], beta=_BETA, margin=_MARGIN,
                            smoothing=c["smoothing"], mean=c["mean"], dloss=state["dloss"] if train else None)
        out = {"loss": got[0], "reward": got[1], "logp": got[2]}
    elif c["op"] == "join":
        form = {"w_post": state["w_post"], "gate": state["gate"], "w_pre": state["w_pre"], "norm": c["norm"], "residual_scale": c["residual"],
                "branch_scale": c["branch"], "rate": c["rate"], "rng": state["rng"]}
        s, z, stats = bz.join(state["x"], state["y"], **form)
        out = {"s": s, "z": z}
        if train:
            back = bz.join_backward(s, state["y"], stats, ds=state["ds"], dz=state["dz"], **form)
            out.update({name: t for name, t in zip(("dx", "dy", "dw_post", "dgate", "dw_pre"), back) if t is not None})
        return out
    else:
        out = {"out": bz.dropout(state["x"], c["rate"], state["rng"])}
        if train:
            out["dx"] = bz.dropout(state["dout"], c["rate"], state["rng"])
        return out
    if train:
        out["dlogits"] = got[-1]
    return out


def work(case):
    e = _SIZE[case["dtype"]]
    train = case["part"] == "train"
    if case["op"] in ("policy", "preference"):
        size, m = case["m"] * case["v"], case["m"]
        # logits, and their gradient; a token and a few numbers a position; exponentials and sums, then two operations an element
        return {"bytes": e * size * (2 if train else 1) + m * 24, "flops": (5 if train else 3) * size}
    size = case["m"] * case["n"]
    if case["op"] == "dropout":
        return {"bytes": e * size * (4 if train else 2), "flops": size * (2 if train else 1)}
    # x, y, s, z; then ds, dz, dx, dy
    vectors = 4 * case["n"] * (1 + (1 if case["post"] else 0) + case["groups"])
    return {"bytes": e * size * (8 if train else 4) + vectors * (2 if train else 1), "flops": (30 if train else 10) * size}


# ---- the definition in 64 bits --------------------------------------------------------------------


def _exact_token(logits, index, temperature):
    """log softmax and the token's entry, None where there is none."""
    log_q = torch.log_softmax(logits.double() / temperature, 1)
    rows = torch.nonzero(index >= 0)[:, 0]
    logp = torch.zeros(logits.shape[0], dtype=torch.float64, device="cuda")
    logp[rows] = log_q[rows, index[rows].long()]
    return log_q, rows, logp


def _exact_gradient(log_q, rows, index, slope):
    """slope * d logp / d logits, zero in the other rows."""
    d = torch.zeros_like(log_q)
    d[rows] = torch.exp(log_q[rows])
    d[rows] *= -slope[rows, None]
    d[rows, index[rows].long()] += slope[rows]
    return d


def _exact_policy(case, s):
    T, kl = case["temperature"], case["kl"]
    log_q, rows, logp = _exact_token(s["logits"], s["index"], T)
    adv, lr = s["advantage"].double(), logp - s["old"].double()
    lo, hi = math.log1p(-_CLIP_LOW), math.log1p(_CLIP_HIGH)
    # min(r A, clip(r) A) is A times r with one side of the clip only: the upper for A >= 0, the lower for A < 0
    used = torch.where(adv >= 0, lr.clamp(max=hi), lr.clamp(min=lo))
    back = s["ref"].double() - logp
    loss = torch.zeros_like(logp)
    loss[rows] = (kl * (torch.expm1(back) - back) - adv * torch.exp(used))[rows]
    out = {"loss": loss, "logp": logp}
    if case["part"] == "train":
        slope = -kl * torch.expm1(back) - adv * torch.exp(lr) * (used == lr)
        out["dlogits"] = _exact_gradient(log_q, rows, s["index"], slope * s["dloss"].double() / T)
    return out


def _exact_preference(case, s):
    pairs, eps = case["pairs"], case["smoothing"]
    log_q, rows, logp = _exact_token(s["logits"], s["index"], 1.0)
    there, starts = s["index"] >= 0, [int(k) for k in s["starts"]]
    gain = torch.where(there, logp - s["ref"].double(), torch.zeros_like(logp))
    counts = [max(1, int(there[a:b].sum())) if case["mean"] else 1 for a, b in zip(starts, starts[1:])]
    reward = torch.stack([_BETA * gain[a:b].sum() / k for a, b, k in zip(starts, starts[1:], counts)])
    h = reward[:pairs] - reward[pairs:] - _MARGIN
    soft = torch.nn.functional.softplus
    out = {"loss": (1 - eps) * soft(-h) + eps * soft(h), "reward": reward, "logp": logp}
    if case["part"] == "train":
        dh = (eps * torch.sigmoid(h) - (1 - eps) * torch.sigmoid(-h)) * s["dloss"].double() * _BETA
        slope = torch.zeros_like(logp)
        for n, (a, b) in enumerate(zip(starts, starts[1:])):
            slope[a:b] = (dh[n] if n < pairs else -dh[n - pairs]) / counts[n]
        out["dlogits"] = _exact_gradient(log_q, rows, s["index"], slope)
    return out


def _exact_keep(rng, m, n, rate):
    """Truth values by 64-bit products in numpy."""
    words = np.empty(((m * n + 7) // 8, 4), np.uint32)
    mask, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    seed, offset = (int(k) for k in rng.tolist())
    for a in range(0, len(words), 1 << 20):
        c = np.arange(a, min(len(words), a + (1 << 20)), dtype=np.uint64)
        one = np.ones_like(c)
        c0, c1, c2, c3 = c & mask, c >> shift, one * np.uint64(offset & 0xFFFFFFFF), one * np.uint64(offset >> 32)
        for r in range(10):
            p, q = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
            key0, key1 = ((seed & 0xFFFFFFFF) + r * 0x9E3779B9) % (1 << 32), ((seed >> 32) + r * 0xBB67AE85) % (1 << 32)
            c0, c1, c2, c3 = (q >> shift) ^ c1 ^ np.uint64(key0), q & mask, (p >> shift) ^ c3 ^ np.uint64(key1), p & mask
        for j, w in enumerate((c0, c1, c2, c3)):
            words[a:a + len(c), j] = w
    # little-endian: the lower half of a word comes first
    bits = words.view(np.uint16).reshape(-1)[: m * n].reshape(m, n)
    return torch.from_numpy(bits >= int(round(rate * 65536))).cuda()


def _exact_dropout(case, s):
    keep = _exact_keep(s["rng"], case["m"], case["n"], case["rate"])
    kept = 65536.0 / (65536 - int(round(case["rate"] * 65536)))
    out = {"out": s["x"].double() * keep * kept}
    if case["part"] == "train":
        out["dx"] = s["dout"].double() * keep * kept
    return out


def _exact_join(case, s):
    """The gradients by automatic differentiation of the definition."""
    m, n, train = case["m"], case["n"], case["part"] == "train"
    leaf = {k: s[k].double().requires_grad_(train) for k in ("x", "y", "w_post", "gate", "w_pre") if s[k] is not None}

    def norm(v, w):
        if case["norm"] == "layer":
            return w * torch.nn.functional.layer_norm(v, (n,), eps=1e-6)
        return w * v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6)

    branch = norm(leaf["y"], leaf["w_post"]) if case["post"] else leaf["y"]
    if case["groups"]:
        branch = (branch.view(case["groups"], -1, n) * leaf["gate"][:, None, :]).view(m, n)
    if case["rate"]:
        branch = branch * _exact_keep(s["rng"], m, n, case["rate"]) * (65536.0 / (65536 - int(round(case["rate"] * 65536))))
    t = case["residual"] * leaf["x"] + case["branch"] * branch
    z = norm(t, leaf["w_pre"])
    out = {"s": t.detach(), "z": z.detach()}
    if train:
        names = list(leaf)
        for k, g in zip(names, torch.autograd.grad((t, z), [leaf[k] for k in names], (s["ds"].double(), s["dz"].double()))):
            out["d" + k] = g
    return out


def exact(case, seed):
    return {"policy": _exact_policy, "preference": _exact_preference, "join": _exact_join, "dropout": _exact_dropout}[case["op"]](case, prepare(case, seed))
