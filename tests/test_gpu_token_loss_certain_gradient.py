"""Gradients of rows whose token is nearly certain: slope / T (1 - p) at the token, which binary32 holds only where 1 - p is not formed from a rounded p.

Where the other tokens are below 2^-25 of the row together its sum is the token's own exponential bit for bit and the entry is 0; the others'
entries are -g p with p within 1e-5, as in test_gpu_token_loss.
"""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from test_gpu_token_loss import DTYPES, HALF_UNIT, TINY, TOL, make, tokens

pytestmark = pytest.mark.gpu


def gradients(x, T):
    """By the fused call, from stats, element by element, and of the preference loss: [(dlogits, upstream times slope)]."""
    m, v = x["logits"].shape
    ones = torch.ones(m, device="cuda")
    _, _, stats, fused = bz.policy(x["logits"], x["index"], ones, temperature=T, dloss=ones)
    out = torch.empty(m, v + 3, dtype=x["logits"].dtype, device="cuda")
    apart = bz.policy(x["logits"], x["index"], ones, temperature=T, dlogits=out[:, 1:1 + v])[3]
    apart_stats = bz.token_loss_backward(x["logits"], x["index"], stats, None, T, dlogits=torch.empty_like(out)[:, 1:1 + v])
    starts = torch.tensor([0, m // 2, m], dtype=torch.int32, device="cuda")
    *_, stats2, pair = bz.preference(x["logits"], x["index"], starts, temperature=T, dloss=torch.ones(1, device="cuda"))
    return [(d, -ones.double().cpu()) for d in (fused, bz.token_loss_backward(x["logits"], x["index"], stats, None, T), apart, apart_stats)] + [(pair, stats2[:, 2].double().cpu())]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v", [(40, 1), (40, 2), (2000, 300), (300, 5000), (8, 70001), (300, 40003)])
def test_certain_tokens_have_no_gradient(m, v, dtype):
    x = make(m, v, dtype, v)
    rows = torch.arange(m, device="cuda")
    x["index"] = (rows * 7 % v).to(torch.int32)
    x["logits"][rows, x["index"].long()] += 64.0
    for T in (1.0, 0.7, 1.3):
        for d, _ in gradients(x, T):
            assert (d[rows, x["index"].long()] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v", [(2000, 300), (300, 5000), (300, 40003)])
def test_likely_tokens(m, v, dtype):
    """1 - p of 10^-1 to 10^-6: its share of the sum is off by a rounding of the sum at each of fewer than 64 additions (72 * 2^-24 with the
    exponentials' own), the rest as everywhere."""
    x = make(m, v, dtype, v)
    rows, host = torch.arange(m, device="cuda"), torch.arange(m)
    x["index"] = (rows * 7 % v).to(torch.int32)
    x["logits"][rows, x["index"].long()] = (rows % 16 + 12).to(dtype)
    _, q, _, at = tokens(x["logits"], x["index"], 1.0)
    for d, g in gradients(x, 1.0):
        want = g * (1 - q[host, at])
        got = d[rows, x["index"].long()].cpu().double()
        assert ((got - want).abs() <= g.abs() * (72 * 2.0 ** -24 + 3 * TOL * (1 - q[host, at])) + HALF_UNIT[dtype] * want.abs() + TINY[dtype]).all()
