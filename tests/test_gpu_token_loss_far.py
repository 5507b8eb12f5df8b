"""bz_policy, bz_preference and their gradient on rows whose largest logit is far from zero: masks of a finite fill, peaks.

Tolerances as in test_gpu_token_loss: exponents are known to 64 * 2^-25 = 2e-6 here too (below the switch to differences the largest's own
exponent is 32 at most).  A token far below the largest has lp = (logit - largest) / T, where the temperature is known to 2^-24 and lp is
rounded once more: three half units of binary32.  Exponentials below 2^-126 become 0 (relative to a whole number: up to 2^-125.5 of the largest);
at T = 0.1 ordinary rows have some, and their gradient is off by that times slope * dloss / T, with |slope * dloss| below 8 here
(advantages below 4.5, dloss below 1.5, ratios below 1.06, kl 0.05): 8 * 10 * 2^-125.5 = 1.4e-36.
"""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from test_gpu_token_loss import F32, HALF_UNIT, TINY, TOL, check_policy, check_preference, gradient, make, near, tokens

pytestmark = pytest.mark.gpu

VANISHED = 1.4e-36


@pytest.fixture(autouse=True)
def least(monkeypatch):
    for dtype in (torch.float32, torch.bfloat16):
        monkeypatch.setitem(TINY, dtype, VANISHED)


FILLS = [-1e9, -1e10, -1e12, -1e20, -1e29, 1e10, 1e20]


def far_rows(m, v, dtype, T):
    """make(), where the first rows are a fill alone, then a fill with one ordinary logit (the token's), then a peak (the token's)."""
    x = make(m, v, dtype, v + 1, T=T)
    x["index"][:3 * len(FILLS)] = 3
    for k, fill in enumerate(FILLS):
        x["logits"][k] = fill
        x["logits"][len(FILLS) + k] = -abs(fill)
        x["logits"][len(FILLS) + k, 3] = 1.0
        x["logits"][2 * len(FILLS) + k, 3] = abs(fill)
    lp = tokens(x["logits"], x["index"], T)[0]
    g = torch.Generator().manual_seed(v)
    x["old"] = (lp + torch.randint(0, 2, (m,), generator=g) * 0.1 - 0.05).float().cuda()
    x["ref"] = (lp + 0.2).float().cuda()
    return x


# rows in a CTA's shared memory, in a cluster's, straight from memory for the loss alone
SIZES = [(30, 500), (30, 70001), (400, 40003)]


@pytest.mark.parametrize("T", [0.1, 0.7, 1.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,v", SIZES)
def test_fills_and_peaks(m, v, dtype, T):
    x = far_rows(m, v, dtype, T)
    d = check_policy(x, T)[3]
    assert torch.isfinite(d).all()
    d = check_preference(x, [0, 9, 15, 22, 30], T=T, beta=0.1, smoothing=0.1)[4]
    assert torch.isfinite(d).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_fills_and_peaks_where_the_gradient_sits_differently(dtype):
    x = far_rows(30, 1001, dtype, 0.7)
    out = torch.empty(30, 1010, dtype=dtype, device="cuda")
    check_policy(x, 0.7, dlogits=out[:, 3:1004])
    check_preference(x, [0, 9, 15, 22, 30], T=0.7, dlogits=out[:, 3:1004])


@pytest.mark.parametrize("T", [0.1, 1.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,v", SIZES)
def test_tokens_far_below_the_largest(m, v, dtype, T):
    x = make(m, v, dtype, 5, T=T)
    x["index"][:2 * len(FILLS)] = 3
    for k, fill in enumerate(FILLS):
        x["logits"][k, 3] = -abs(fill)
        x["logits"][len(FILLS) + k, 7] = abs(fill)
    n = 2 * len(FILLS)
    ones = torch.ones(m, device="cuda")
    _, logp, stats, d = bz.policy(x["logits"], x["index"], ones, temperature=T, dloss=ones)
    lp, q, there, at = tokens(x["logits"][:n], x["index"][:n], T)
    assert near(logp[:n], lp, TOL + 3 * F32 * lp.abs())
    one = torch.ones(n, dtype=torch.float64)
    want, bound = gradient(q, there, at, -one, one, one, T)
    bound = bound + HALF_UNIT[dtype] * want.abs() + TINY[dtype]
    assert near(d[:n], want, bound) and near(bz.token_loss_backward(x["logits"], x["index"], stats, None, T)[:n], want, bound)


@pytest.mark.parametrize("fill,T", [(-1e10, 100.0), (-1e10, 10.0), (1e10, 20.0), (-3e9, 3.0), (1.6e9, 1.0)])
def test_neighbours_far_from_zero(fill, T):
    """Logits a few units of binary32 apart, a row's sum made of several: on both sides of the switch from whole numbers to differences."""
    m, v = 64, 3001
    g = torch.Generator().manual_seed(1)
    x = make(m, v, torch.float32, 1, T=T)
    start = torch.full((m, v), fill)
    unit = torch.nextafter(start.abs(), torch.full_like(start, float("inf"))) - start.abs()
    x["logits"].copy_(start + unit * torch.randint(0, 5, (m, v), generator=g))
    x["index"] = torch.randint(0, v, (m,), generator=g, dtype=torch.int32).cuda()
    lp = tokens(x["logits"], x["index"], T)[0]
    x["old"], x["ref"] = (lp + 0.05).float().cuda(), (lp - 0.1).float().cuda()
    ones = torch.ones(m, device="cuda")
    _, logp, stats, d = bz.policy(x["logits"], x["index"], ones, temperature=T, dloss=ones)
    lp, q, there, at = tokens(x["logits"], x["index"], T)
    assert near(logp, lp, TOL + 3 * F32 * lp.abs())
    one = torch.ones(m, dtype=torch.float64)
    want, bound = gradient(q, there, at, -one, one, one, T)
    # a probability's exponent is off by the temperature's 2^-24 too
    bound = bound + 3 * F32 * ((q.clamp(min=1e-300).log().abs() + 3) * q / T) + F32 * want.abs() + TINY[torch.float32]
    assert near(d, want, bound) and near(bz.token_loss_backward(x["logits"], x["index"], stats, None, T), want, bound)


@pytest.mark.parametrize("T", [1e-3, 1e-6, 1e-9, 1e-30])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,v", SIZES)
def test_low_temperatures(m, v, dtype, T):
    """Ordinary logits, whose exponents a low temperature takes as far: nearly all of a row is its largest token's.  The temperature reaches the
    kernel as a binary32 number, and exponentials below 2^-126 become 0."""
    T = float(torch.tensor(T))
    x = make(m, v, dtype, 9, T=T)
    x["index"][::2] = x["logits"][::2].float().argmax(1).int()
    ones = torch.ones(m, device="cuda")
    _, logp, stats, d = bz.policy(x["logits"], x["index"], ones, temperature=T, dloss=ones)
    lp, q, there, at = tokens(x["logits"], x["index"], T)
    assert near(logp, lp, TOL + 3 * F32 * lp.abs()) and (logp <= 0).all()
    one = torch.ones(m, dtype=torch.float64)
    want, bound = gradient(q, there, at, -one, one, one, T)
    # a probability's exponent is off by the temperature's 2^-24 too
    bound = bound + 3 * F32 * q.clamp(min=1e-300).log().abs() * q / T + HALF_UNIT[dtype] * want.abs() + TINY[dtype] + 2.0 ** -125 / T
    most = torch.finfo(dtype).max * (1 + HALF_UNIT[dtype])      # beyond it the rounded value is an infinity
    want = torch.where(want.abs() > most, want.sign() * float("inf"), want)
    assert near(d, want, bound) and near(bz.token_loss_backward(x["logits"], x["index"], stats, None, T), want, bound)
