"""The operators of a fine-tuning step as they are used together: norms, gates and dropout around the blocks, the policy and the
preference loss, file gradients voted on and applied."""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from paper_2010_04902_b200 import worker_step as ws
from test_gpu_dropout import kept

pytestmark = pytest.mark.gpu


def _one_file(kind, seed=0):
    w = ws.initial(seed, ws.TUNED)
    views = ws.views(w, ws.TUNED)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for name in ws.JOINS:      # not all alike, so that a gradient in the wrong place shows
        views[name].add_(torch.randn(views[name].shape, generator=g, device="cuda") * 0.1)
    views["table"].normal_(0.0, 0.5, generator=g)
    tokens, objective = ws.sampled_file(kind, ws.Teacher(), g)
    rng = torch.tensor([[seed + 7, k] for k in range(3)], device="cuda")
    return w, ws.tuned_weights(w), tokens, objective, rng


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_copies_of_a_file_are_identical_and_the_vote_keeps_them(kind):
    _, weights, tokens, objective, rng = _one_file(kind)
    replicas = torch.empty(3, 1, ws.TUNED_SIZE, device="cuda")
    for k in range(3):
        ws.tuned_gradient(weights, tokens, objective, rng, 0.1, replicas[k, 0])
    assert torch.equal(replicas[0], replicas[1]) and torch.equal(replicas[0], replicas[2])
    honest = replicas[0, 0].clone()
    assert torch.isfinite(honest).all() and float(honest.abs().max()) > 0
    replicas[1] *= -100.0
    assert torch.equal(bz.vote(replicas)[0], honest)
    ws.tuned_gradient(weights, tokens, objective, rng + 100, 0.1, replicas[0, 0])
    assert not torch.equal(replicas[0, 0], honest)      # another mask, another gradient


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_gradient_agrees_with_automatic_differentiation(kind):
    """The whole step against torch's own differentiation in binary32 of the same (bfloat16-valued) weights and the same masks.  The step
    rounds activations and gradients to bfloat16 (2^-9 relative each) some twenty times on the way: 4 % of each gradient's norm."""
    rate = 0.2
    _, weights, tokens, objective, rng = _one_file(kind, 3)
    row = torch.empty(ws.TUNED_SIZE, device="cuda")
    ws.tuned_gradient(weights, tokens, objective, rng, rate, row)
    p = {k: v.float().clone().requires_grad_(True) for k, v in weights.items()}
    n, t = tokens.shape
    d, width = ws.WIDTH // ws.HEADS, ws.WIDTH
    scale = 65536 / (65536 - round(rate * 65536))
    drop = lambda x, k: x * kept(rng[k].tolist(), x.numel(), rate).view(x.shape).cuda() * scale  # noqa: E731
    heads = lambda x: x.view(n, t, ws.HEADS, d).transpose(1, 2)  # noqa: E731
    norm = lambda x, w: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w  # noqa: E731
    x = p["embedding"][tokens.reshape(-1)]
    a = norm(x, p["norm_in"])
    rel = torch.arange(t, device="cuda")[None, :] - torch.arange(t, device="cuda")[:, None]
    far = torch.clamp(-rel, min=0)
    exact = ws.BUCKETS // 2
    log = exact + (torch.log(far.double().clamp(min=1) / exact) / torch.log(torch.tensor(ws.DISTANCE / exact, dtype=torch.float64)) *
                   (ws.BUCKETS - exact) + 1e-9).long().clamp(max=ws.BUCKETS - exact - 1)
    bias = p["table"][torch.where(far < exact, far, log)].permute(2, 0, 1)
    scores = heads(a @ p["wq"].T) @ heads(a @ p["wk"].T).transpose(2, 3) * d ** -0.5 + bias
    probs = drop(torch.softmax(scores.masked_fill(rel > 0, float("-inf")), -1), 0)
    out = (probs @ heads(a @ p["wv"].T)).transpose(1, 2).reshape(n * t, width) @ p["wo"].T
    s1 = x + drop(p["gate_attention"] * norm(out, p["norm_attention"]), 1)
    y = norm(s1, p["norm_block"])
    f = (torch.nn.functional.gelu(y @ p["w_gate"].T, approximate="tanh") * (y @ p["w_up"].T)) @ p["w_down"].T
    s2 = s1 + drop(p["gate_ffn"] * norm(f, p["norm_ffn"]), 2)
    logits = norm(s2, p["norm_head"]) @ p["head"].T
    with torch.no_grad():
        _, dlogits = objective(logits.detach())
    logits.backward(dlogits)
    for name, got in ws.views(row, ws.TUNED).items():
        g = p[name].grad
        assert float((got - g).norm()) <= 0.04 * float(g.norm()), name


@pytest.mark.parametrize("kind,byzantine", [("policy", 3), ("preference", 0)])
def test_it_runs(kind, byzantine):
    losses = ws.tune(3, byzantine, kind, same_bits=True)
    assert len(losses) == 3 and all(abs(v) < 1e3 for v in losses)
