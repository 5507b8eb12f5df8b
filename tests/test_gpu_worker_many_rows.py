"""Rows enough that every CTA of the worker's row kernels takes many of them, one behind the other: the next row's loads in
flight, the alternating sets of partial results, diagonals summed over rows, rings that go round.  Against the formulas in 64
bits, formed on the GPU for whole tensors at a time.  And the operators as recorded into a CUDA graph.

Tolerances as in the tests of single rows (an exponent's argument below 40 is known to 7e-6, so p and q to 1e-5 relative;
half a unit of the type on top); a table gradient is a sum of at most 2^11 additions one after the other (64 rows of 16 elements
a lane, then lanes, warps and CTAs), each off by 2^-24 of the terms' sizes so far.
"""
import math

import pytest
import torch

from paper_2010_04902_b200 import binding as bz

pytestmark = pytest.mark.gpu

HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}
TOL = 1e-5
TABLE_TOL = 2 * TOL + 2.0 ** 11 * 2.0 ** -24


def bucket(rel, buckets, distance, both):
    nb = buckets // 2 if both else buckets
    n, e = (abs(rel) if both else max(-rel, 0)), nb // 2
    c = n if n < e else e + max(t for t in range(nb - e) if n ** (nb - e) >= e ** (nb - e - t) * distance ** t)
    return c + nb if both and rel > 0 else c


def reference(scores, table, distance, both, causal, k_len, q_start, dprobs):
    """(p, log-sum, dz, size of dz's terms, dtable, size of its terms), batch entry by batch entry."""
    b, h, tq, tk = scores.shape
    near = [bucket(r, table.shape[0], distance, both) for r in range(-distance, distance + 1)]
    near = torch.tensor(near, device="cuda")
    dt, dt_size = torch.zeros(table.shape, dtype=torch.float64, device="cuda"), torch.zeros(table.shape, dtype=torch.float64, device="cuda")
    for ib in range(b):
        i, j = torch.arange(tq, device="cuda")[:, None], torch.arange(tk, device="cuda")[None]
        rel = j - i - (0 if q_start is None else int(q_start[ib]))
        seen = (j < (tk if k_len is None else int(k_len[ib]))) & ((rel <= 0) | (not causal))
        kind = near[rel.clamp(-distance, distance) + distance]
        z = (scores[ib].double() + table.double()[kind].permute(2, 0, 1)).masked_fill_(~seen, -math.inf)
        lse = torch.logsumexp(z, -1)
        p = torch.where(torch.isinf(lse)[..., None], torch.zeros_like(z), torch.exp(z - lse[..., None]))
        dp = dprobs[ib].double()
        dz = p * (dp - (p * dp).sum(-1, keepdim=True))
        size = p * (dp.abs() + (p * dp.abs()).sum(-1, keepdim=True))
        dt.index_add_(0, kind.reshape(-1), dz.reshape(h, -1).T)
        dt_size.index_add_(0, kind.reshape(-1), size.reshape(h, -1).T)
        yield p, lse, dz, size
    yield dt, dt_size


def tensor(shape, dtype, seed, sigma, pad):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape[:-1], shape[-1] + pad, generator=g, device="cuda") * sigma).to(dtype)[..., :shape[-1]]


@pytest.mark.parametrize("b,h,tq,tk,dtype,how", [
    (4, 16, 1024, 40, torch.bfloat16, {}), (4, 16, 1024, 77, torch.float16, {"pad": 3}), (4, 16, 1024, 300, torch.bfloat16, {"ragged": True}),
    (2, 16, 1024, 500, torch.float32, {"causal": True}), (2, 16, 1024, 512, torch.float32, {}), (2, 16, 1024, 1024, torch.bfloat16, {}),
    (4, 8, 1024, 1024, torch.bfloat16, {"causal": True}), (2, 16, 500, 1500, torch.float16, {"causal": True, "ragged": True}),
    (1, 16, 400, 2048, torch.bfloat16, {}), (1, 16, 300, 4099, torch.bfloat16, {"pad": 1, "causal": True}), (1, 8, 300, 4096, torch.float32, {}),
    (1, 8, 300, 9000, torch.float16, {"ragged": True}), (1, 8, 200, 17001, torch.bfloat16, {"pad": 7}), (2, 16, 512, 260, torch.bfloat16, {"apart": 5}),
    (1, 8, 300, 5000, torch.float32, {"apart": 1, "causal": True}), (2, 16, 512, 700, torch.bfloat16, {"distance": 400, "both": False})])
def test_softmax_of_many_rows(b, h, tq, tk, dtype, how):
    """`pad`: all rows that much longer in memory; `apart`: those of dprobs alone."""
    distance, both, causal = how.get("distance", 128), how.get("both", not how.get("causal")), how.get("causal", False)
    pad = how.get("pad", 0)
    scores = tensor((b, h, tq, tk), dtype, tk, 2.0, pad)
    dprobs = tensor((b, h, tq, tk), dtype, tk + 1, 1.0, how.get("apart", pad))
    table = torch.randn(32, h, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    k_len = torch.tensor([tk - 37 * i - 5 for i in range(b)], dtype=torch.int32, device="cuda") if how.get("ragged") else None
    q_start = torch.tensor([tk - tq + 3 * i for i in range(b)], dtype=torch.int32, device="cuda") if causal and tk > tq else None
    form = dict(max_distance=distance, bidirectional=both, causal=causal, k_len=k_len, q_start=q_start)
    p, stats = bz.bias_softmax(scores, table, **form)
    ds, dt = bz.bias_softmax_backward(scores, table, stats, dprobs, **form)
    want = list(range(b))
    ref = reference(scores, table, distance, both, causal, k_len, q_start, dprobs)
    hu, tiny = HALF_UNIT[dtype], TINY[dtype]
    for ib in want:
        wp, lse, dz, size = next(ref)
        assert ((p[ib].double() - wp).abs() <= wp * (TOL + hu) + tiny).all()
        got = stats[ib, ..., 0].double() + torch.log(stats[ib, ..., 1].double())
        assert ((got == lse) | ((got - lse).abs() <= TOL)).all()
        assert ((ds[ib].double() - dz).abs() <= 2 * TOL * size + hu * dz.abs() + tiny).all()
        del wp, dz, size
    wdt, dt_size = next(ref)
    assert ((dt.double() - wdt).abs() <= TABLE_TOL * dt_size + 1e-30).all()
    for _ in range(5):
        p2, stats2 = bz.bias_softmax(scores, table, **form)
        ds2, dt2 = bz.bias_softmax_backward(scores, table, stats, dprobs, **form)
        assert torch.equal(p, p2) and torch.equal(stats, stats2) and torch.equal(ds, ds2) and torch.equal(dt, dt2)


@pytest.mark.parametrize("m,v,t,dtype,pad", [(1900, 8200, 16, torch.bfloat16, 0), (1900, 9001, 40, torch.float32, 3), (1800, 32128, 64, torch.bfloat16, 0),
                                             (1790, 33003, 50, torch.float16, 5), (1777, 40001, 5, torch.bfloat16, 0)])
def test_distillation_of_many_positions(m, v, t, dtype, pad):
    """At least six rows a CTA of the ring, held and read twice."""
    g = torch.Generator(device="cuda").manual_seed(v)
    logits = tensor((m, v), dtype, v, 2.5, pad)
    teacher = torch.randn(m, t, generator=g, device="cuda") * 3
    index = torch.randint(0, v, (m, t), generator=g, device="cuda", dtype=torch.int32)
    index[::7, t // 2:] = -1
    index[5::50] = -1
    index[11::64, 1:] = index[11::64, :1]
    dloss = torch.rand(m, generator=g, device="cuda") + 0.5
    T = 2.0
    loss, stats, d = bz.distill(logits, teacher, index, T, dloss=dloss)
    alone, stats2 = bz.distill(logits, teacher, index, T)
    back = bz.distill_backward(logits, teacher, index, stats, dloss, T)
    assert torch.equal(stats, stats2) and torch.equal(loss, alone)
    hu = HALF_UNIT[dtype]
    for lo in range(0, m, 400):
        part = slice(lo, min(lo + 400, m))
        s = logits[part].double() / T
        log_q = s - torch.logsumexp(s, 1, keepdim=True)
        kept = index[part] >= 0
        z = (teacher[part].double() / T).masked_fill(~kept, -math.inf)
        log_p = torch.where(kept, z - torch.logsumexp(z, 1, keepdim=True), torch.zeros_like(z))
        p = torch.where(kept, torch.exp(log_p), torch.zeros_like(z))
        at = index[part].long().clamp(min=0)
        want = T * T * (p * (log_p - log_q.gather(1, at))).sum(1)
        assert ((loss[part].double() - want).abs() <= TOL * T * T + TOL * want.abs()).all()
        q = torch.exp(log_q) * kept.any(1)[:, None]
        named = torch.zeros_like(q).scatter_add_(1, at, p)
        scale = (dloss[part].double() * T)[:, None]
        grad, size = scale * (q - named), scale * (q + named)
        bound = 2 * TOL * size + hu * grad.abs() + TINY[dtype]
        assert ((d[part].double() - grad).abs() <= bound).all() and ((back[part].double() - grad).abs() <= bound).all()
        lse = stats[part, 0].double() / T + torch.log(stats[part, 1].double())
        assert ((lse - torch.logsumexp(s, 1)).abs() <= TOL).all()


def test_calls_in_a_graph():
    """Each call recorded with its outputs and workspaces given, then replayed on other inputs: the same bits as a direct call."""
    def data(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        return {"x": r(300, 264).to(torch.bfloat16), "few": r(3, 264).to(torch.bfloat16), "off": r(40, 261).to(torch.bfloat16), "wg": r(136, 264).to(torch.bfloat16),
                "wu": r(136, 264).to(torch.bfloat16), "wo": r(50, 261).to(torch.bfloat16), "dh": r(300, 136).to(torch.bfloat16),
                "scores": r(2, 4, 50, 300).to(torch.bfloat16), "dprobs": r(2, 4, 50, 300).to(torch.bfloat16), "table": r(32, 4),
                "logits": r(200, 9000).to(torch.bfloat16), "short": r(20, 999), "teacher": r(200, 9), "dloss": r(200),
                "index": torch.randint(0, 999, (200, 9), generator=g, device="cuda", dtype=torch.int32)}

    def steps(d, o):
        bz.glu(d["few"], d["wg"], d["wu"], h=o["few"])
        bz.glu(d["off"], d["wo"], d["wo"], h=o["off"], workspace=o["ws0"])
        bz.glu(d["x"], d["wg"], d["wu"], h=o["h"], preact=o["preact"])
        bz.glu_backward(d["x"], d["wg"], d["wu"], o["preact"], d["dh"], dx=o["dx"], dw_gate=o["dg"], dw_up=o["du"], workspace=o["ws1"])
        bz.bias_softmax(d["scores"], d["table"], probs=o["probs"], stats=o["stats"])
        bz.bias_softmax_backward(d["scores"], d["table"], o["stats"], d["dprobs"], dscores=o["ds"], dtable=o["dt"], workspace=o["ws2"])
        bz.distill(d["logits"], d["teacher"], d["index"], 2.0, dloss=d["dloss"], loss=o["loss"], stats=o["lstats"], dlogits=o["dl"])
        bz.distill(d["short"], d["teacher"][:20], d["index"][:20], 2.0, loss=o["loss2"], stats=o["lstats2"])
        bz.distill_backward(d["short"], d["teacher"][:20], d["index"][:20], o["lstats2"], temperature=2.0, dlogits=o["dl2"])

    def outputs():
        e = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        f, u = torch.float32, torch.uint8
        return {"few": e(3, 136), "off": e(40, 50), "h": e(300, 136), "preact": e(2, 300, 136, t=f), "dx": e(300, 264), "dg": e(136, 264, t=f), "du": e(136, 264, t=f),
                "probs": e(2, 4, 50, 300), "stats": e(2, 4, 50, 2, t=f), "ds": e(2, 4, 50, 300), "dt": e(32, 4, t=f), "loss": e(200, t=f), "lstats": e(200, 2, t=f),
                "dl": e(200, 9000), "loss2": e(20, t=f), "lstats2": e(20, 2, t=f), "dl2": e(20, 999, t=f),
                "ws0": e(bz.glu_workspace_bytes(40, 50, 261), t=u), "ws1": e(bz.glu_workspace_bytes(300, 136, 264, backward=True), t=u),
                "ws2": e(bz.lib().bz_bias_softmax_workspace_bytes(2, 4, 50, 300, 32), t=u)}

    d, o = data(1), outputs()
    steps(d, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(d, o)
    for seed in (2, 3):
        new, want = data(seed), outputs()
        for k, v in new.items():
            d[k].copy_(v)
        graph.replay()
        steps(new, want)
        torch.cuda.synchronize()
        for k in want:
            if not k.startswith("ws"):
                assert torch.equal(o[k], want[k]), k
