"""The worker's operators as they are used together: file gradients of a small model, voted on and applied."""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from paper_2010_04902_b200 import worker_step as ws

pytestmark = pytest.mark.gpu


def _one_file(seed=0):
    w = ws.initial(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    tokens = torch.randint(0, ws.VOCAB, (ws.SEQUENCES, ws.LENGTH), generator=g, device="cuda")
    top, index = ws.Teacher()(tokens)
    return w, {**ws.views(w.to(torch.bfloat16)), "table": ws.views(w)["table"]}, tokens, top, index


def test_copies_of_a_file_are_identical_and_the_vote_keeps_them():
    _, weights, tokens, top, index = _one_file()
    replicas = torch.empty(3, 1, ws.SIZE, device="cuda")
    for k in range(3):
        ws.file_gradient(weights, tokens, top, index, replicas[k, 0])
    assert torch.equal(replicas[0], replicas[1]) and torch.equal(replicas[0], replicas[2])
    honest = replicas[0, 0].clone()
    assert torch.isfinite(honest).all() and float(honest.abs().max()) > 0
    replicas[1] *= -100.0
    assert torch.equal(bz.vote(replicas)[0], honest)


def test_gradient_agrees_with_automatic_differentiation():
    """The whole step against torch's own differentiation in binary32 of the same (bfloat16-valued) weights.  The step rounds
    activations and gradients to bfloat16 (2^-9 relative each) some ten times on the way: 3 % of each gradient's norm."""
    _, weights, tokens, top, index = _one_file(3)
    row = torch.empty(ws.SIZE, device="cuda")
    loss = ws.file_gradient(weights, tokens, top, index, row)
    p = {k: v.float().clone().requires_grad_(True) for k, v in weights.items()}
    n, t = tokens.shape
    d = ws.WIDTH // ws.HEADS
    heads = lambda x: x.view(n, t, ws.HEADS, d).transpose(1, 2)  # noqa: E731
    x = p["embedding"][tokens.reshape(-1)]
    rel = torch.arange(t, device="cuda")[None, :] - torch.arange(t, device="cuda")[:, None]
    far = torch.clamp(-rel, min=0)
    exact = ws.BUCKETS // 2
    log = exact + (torch.log(far.double().clamp(min=1) / exact) / torch.log(torch.tensor(ws.DISTANCE / exact, dtype=torch.float64)) *
                   (ws.BUCKETS - exact) + 1e-9).long().clamp(max=ws.BUCKETS - exact - 1)
    bias = p["table"][torch.where(far < exact, far, log)].permute(2, 0, 1)
    scores = heads(x @ p["wq"].T) @ heads(x @ p["wk"].T).transpose(2, 3) * d ** -0.5 + bias
    probs = torch.softmax(scores.masked_fill(rel > 0, float("-inf")), -1)
    y = x + (probs @ heads(x @ p["wv"].T)).transpose(1, 2).reshape(n * t, -1) @ p["wo"].T
    h = torch.nn.functional.gelu(y @ p["w_gate"].T, approximate="tanh") * (y @ p["w_up"].T)
    logits = (y + h @ p["w_down"].T) @ p["head"].T / 2.0
    log_q, q = torch.log_softmax(logits, 1), torch.softmax(top / 2.0, 1)
    want = 4.0 * (q * (torch.log(q) - log_q.gather(1, index.long()))).sum(1)
    want.mean().backward()
    assert torch.allclose(loss, want, rtol=0.02, atol=0.05)
    for name, got in ws.views(row).items():
        g = p[name].grad
        assert float((got - g).norm()) <= 0.03 * float(g.norm()), name


@pytest.mark.parametrize("byzantine", [0, 3])
def test_it_learns(byzantine):
    losses = ws.train(20, byzantine, eta=2.0, same_bits=True)
    assert losses[-1] < 0.97 * losses[0]
    assert sum(losses[-5:]) < sum(losses[:5])


def test_workspaces_are_checked():
    """A workspace in host memory is refused before any launch; one of another type counts by its bytes."""
    x, w = torch.randn(40, 9, device="cuda").to(torch.bfloat16), torch.randn(6, 9, device="cuda").to(torch.bfloat16)
    dh, preact = torch.randn(40, 6, device="cuda").to(torch.bfloat16), torch.empty(2, 40, 6, device="cuda")
    scores, table = torch.randn(1, 2, 3, 8, device="cuda"), torch.randn(32, 2, device="cuda")
    _, stats = bz.bias_softmax(scores, table)
    h = bz.glu(x, w, w, preact=preact)
    calls = [(lambda ws: bz.glu(x, w, w, workspace=ws), bz.glu_workspace_bytes(40, 6, 9)),
             (lambda ws: bz.glu_backward(x, w, w, preact, dh, workspace=ws), bz.glu_workspace_bytes(40, 6, 9, backward=True)),
             (lambda ws: bz.bias_softmax_backward(scores, table, stats, scores, workspace=ws), bz.lib().bz_bias_softmax_workspace_bytes(1, 2, 3, 8, 32)),
             (lambda ws: bz.pairdist(scores.view(6, 8), workspace=ws), bz.workspace_bytes(bz.OP_PAIRDIST, 0, 6, 8))]
    for call, size in calls:
        n0 = bz.kernel_launch_count()
        with pytest.raises(TypeError, match="workspace"):
            call(torch.empty(size, dtype=torch.uint8))
        with pytest.raises(TypeError, match="workspace"):
            call(torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2])
        with pytest.raises(bz.BzError):
            call(torch.empty(max(size - 256, 1) // 4, device="cuda"))
        assert bz.kernel_launch_count() == n0
        call(torch.empty((size + 3) // 4, device="cuda"))
    assert torch.equal(bz.glu(x, w, w, workspace=torch.empty(4096, device="cuda")), h)
