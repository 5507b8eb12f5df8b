"""Log-probabilities of tokens that are nearly certain: never above 0, and 0 where binary32 has nothing between.

Relative to its own exponential a row's sum is 1 + the others.  Each addition on the way of that 1 rounds by half a unit of the sum at
most, 2^-24 of it, and there are fewer than 64 (a thread's groups of words, then lanes, warps, CTAs); the exponentials are off by 4 half units:
lp is within 72 * 2^-24 and half a unit of its own.  Others that are below 2^-25 together leave the sum as it is: lp is 0.
"""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from test_gpu_token_loss import DTYPES, F32, TOL, make, near, tokens

pytestmark = pytest.mark.gpu

SIZES = [(40, 1), (40, 2), (2000, 300), (300, 5000), (8, 70001), (300, 70001)]


def logp_of(x, T, which):
    m, v = x["logits"].shape
    ones = torch.ones(m, device="cuda")
    if which == "policy":
        return bz.policy(x["logits"], x["index"], ones, temperature=T)[1]
    if which == "gradient":
        return bz.policy(x["logits"], x["index"], ones, temperature=T, dloss=ones)[1]
    if which == "differently":      # a gradient that sits differently: element by element
        out = torch.empty(m, v + 3, dtype=x["logits"].dtype, device="cuda")
        return bz.policy(x["logits"], x["index"], ones, temperature=T, dlogits=out[:, 1:1 + v])[1]
    return bz.preference(x["logits"], x["index"], torch.tensor([0, m // 2, m], dtype=torch.int32, device="cuda"), temperature=T)[2]


@pytest.mark.parametrize("which", ["policy", "gradient", "differently", "preference"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v", SIZES)
def test_one_logit_far_above_the_others(m, v, dtype, which):
    x = make(m, v, dtype, v)
    rows = torch.arange(m, device="cuda")
    x["index"] = (rows * 7 % v).to(torch.int32)
    x["logits"][rows, x["index"].long()] += 64.0
    for T in (1.0, 0.7, 1.3):
        assert (logp_of(x, T, which) == 0).all()


def test_two_logits():
    x = make(1, 2, torch.float32, 0)
    x["index"][0] = 0
    for far in (30.0, 100.0, 1e4):
        x["logits"][0, 0], x["logits"][0, 1] = 0.0, -far
        for which in ("policy", "gradient", "preference"):
            assert float(logp_of(x, 1.0, which)[0]) == 0.0


@pytest.mark.parametrize("which", ["policy", "gradient", "differently", "preference"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v", [(2000, 300), (300, 5000), (300, 70001)])
def test_between_likely_and_certain(m, v, dtype, which):
    x = make(m, v, dtype, v)
    rows = torch.arange(m, device="cuda")
    x["index"] = (rows * 7 % v).to(torch.int32)
    x["logits"][rows, x["index"].long()] = (torch.arange(m, device="cuda") % 32 + 4).to(dtype)
    lp, q, _, at = tokens(x["logits"], x["index"], 1.0)
    got = logp_of(x, 1.0, which)
    p = q[torch.arange(m), at]
    assert (got <= 0).all()
    likely = p > 0.6
    assert int(likely.sum()) > m // 4
    assert near(got[likely.cuda()], lp[likely], 72 * F32 + F32 * lp[likely].abs())
    assert near(got, lp, TOL + F32 * lp.abs())
