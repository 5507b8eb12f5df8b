"""bz_policy, bz_preference and their gradient against the formulas in 64 bits.

Tolerances.  With |logits| / T below 40 an exponent's argument is known to about 40 * 1.44 * 2^-23 = 7e-6, so probabilities are
within 1e-5 relative and lp within 1e-5, and half a unit of binary32.  A loss then moves by its slope times that, a slope by its own
derivative times that; dlogits = dloss slope / T ([c == a] - p) within these shares, and half a unit of its type.
"""
import math

import pytest
import torch

from paper_2010_04902_b200 import binding as bz

pytestmark = pytest.mark.gpu

HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}
TOL = 1e-5
F32 = 2.0 ** -24
LOW, HIGH = 0.2, 0.28


def tokens(logits, index, T):
    """lp, softmax, which rows have a token (64 bits, on the host)."""
    z = logits.detach().cpu().double() / T
    v = z.shape[1]
    there = (index.cpu() >= 0) & (index.cpu() < v)
    at = torch.where(there, index.cpu().long(), torch.zeros(1, dtype=torch.long))
    # the largest goes first: beside a type's lowest value 64 bits would not hold the logarithm
    top = z.amax(1, keepdim=True)
    z = z - torch.where(top == -math.inf, torch.zeros_like(top), top)
    lse = torch.logsumexp(z, 1)
    log_q = torch.where(lse[:, None] == -math.inf, torch.full_like(z, -math.inf), z - lse[:, None])
    lp = torch.where(there, log_q[torch.arange(len(at)), at], torch.zeros(1, dtype=torch.float64))
    return lp, torch.exp(log_q), there, at


def gradient(q, there, at, slope, bend, dloss, T):
    """(dlogits, what it may be off by but for the last rounding)."""
    hot = torch.zeros_like(q)
    hot[torch.arange(len(at)), at] = 1.0
    g = torch.where(there, slope * dloss / T, torch.zeros(1, dtype=torch.float64))
    on = (g != 0)[:, None]
    d = torch.where(on, g[:, None] * (hot - q), torch.zeros_like(q))
    size = torch.where(on, ((slope.abs() + bend.abs()) * dloss.abs() / T)[:, None] * (hot + q), torch.zeros_like(q))
    return d, 3 * TOL * size


def policy_reference(lp, old, ref, adv, kl):
    r = torch.exp(lp - old) if old is not None else torch.ones_like(lp)
    held = ((adv > 0) & (r > 1 + HIGH)) | ((adv < 0) & (r < 1 - LOW))
    used = torch.where(held, r.clamp(1 - LOW, 1 + HIGH), r)
    loss = torch.where(adv == 0, torch.zeros_like(lp), -used * adv)
    slope = torch.where(held | (adv == 0), torch.zeros_like(lp), -r * adv)
    bend = slope.clone()
    if kl:
        d = ref - lp
        loss = loss + kl * (torch.exp(d) - d - 1)
        slope = slope - kl * torch.expm1(d)
        bend = bend.abs() + kl * torch.exp(d)
    return loss, torch.where(lp == -math.inf, torch.zeros_like(lp), slope), bend


def near(got, want, tol):
    got = got.cpu().double()
    return bool(((got == want) | ((got - want).abs() <= tol) | (got.isnan() & want.isnan())).all())


def make(m, v, dtype, seed, pad=0, T=1.0):
    g = torch.Generator().manual_seed(seed)
    full = torch.empty(m, v + pad, dtype=dtype, device="cuda")
    full[:, :v] = (torch.randn(m, v, generator=g) * 2.5).to(dtype).cuda()
    logits = full[:, :v]
    index = torch.randint(0, v, (m,), generator=g, dtype=torch.int32)
    index[torch.rand(m, generator=g) < 0.15] = -1
    lp = tokens(logits, index, T)[0]
    moved = torch.randn(m, generator=g).double() * 0.3
    for border in (math.log(1 - LOW), math.log(1 + HIGH)):     # a ratio within rounding of a border may fall on either side
        moved = torch.where((moved - border).abs() < 1e-3, moved + 4e-3, moved)
    return {"logits": logits, "index": index.cuda(), "old": (lp - moved).float().cuda(), "ref": (lp + torch.randn(m, generator=g) * 0.3).float().cuda(),
            "adv": torch.randn(m, generator=g).cuda(), "dloss": (torch.rand(m, generator=g) + 0.5).cuda()}


def check_policy(x, T=1.0, kl=0.05, on_policy=False, dlogits=None):
    old = None if on_policy else x["old"]
    form = {"old_logp": old, "ref_logp": x["ref"], "kl": kl, "clip_low": LOW, "clip_high": HIGH, "temperature": T}
    lp, q, there, at = tokens(x["logits"], x["index"], T)
    d64 = lambda t: None if t is None else t.cpu().double()  # noqa: E731
    want, slope, bend = policy_reference(lp, d64(old), d64(x["ref"]), d64(x["adv"]), kl)
    want = torch.where(there, want, torch.zeros_like(want))
    loss, logp, stats, d = bz.policy(x["logits"], x["index"], x["adv"], **form, dloss=x["dloss"], dlogits=dlogits)
    assert near(logp, lp, TOL + F32 * lp.abs())
    reach = slope.abs() + bend.abs()
    # the clip's borders reach the kernel as binary32 numbers: another half unit
    assert near(loss, want, TOL * reach + 2 * F32 * want.abs())
    wd, bound = gradient(q, there, at, slope, bend, d64(x["dloss"]), T)
    bound = bound + HALF_UNIT[d.dtype] * wd.abs() + TINY[d.dtype]
    # beyond the type's range the rounded value is an infinity
    wd = torch.where(wd.abs() > torch.finfo(d.dtype).max * (1 + HALF_UNIT[d.dtype]), wd.sign() * math.inf, wd)
    assert near(d, wd, bound)
    only = bz.policy(x["logits"], x["index"], x["adv"], **form)
    assert len(only) == 3 and near(only[0], want, TOL * reach + 2 * F32 * want.abs()) and near(only[1], lp, TOL + F32 * lp.abs())
    assert near(bz.token_loss_backward(x["logits"], x["index"], stats, x["dloss"], T), wd, bound)
    return loss, logp, stats, d


DTYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v,T,kl", [(1, 1, 1.0, 0.1), (3, 2, 2.0, 0.0), (5, 33, 1.0, 0.05), (7, 1001, 0.7, 0.05), (4, 1024, 1.0, 0.1), (2, 8193, 1.5, 0.02),
                                      (2, 32768, 1.0, 0.05), (2, 32771, 1.0, 0.05), (3, 70001, 0.7, 0.05), (2, 200003, 1.0, 0.0), (1, 300001, 1.0, 0.05)])
def test_policy_matches(m, v, T, kl, dtype):
    check_policy(make(m, v, dtype, v, T=T), T, kl)


@pytest.mark.parametrize("dtype,m,v,pad", [(torch.bfloat16, 500, 8200, 0), (torch.bfloat16, 700, 8201, 0), (torch.float32, 400, 4111, 1), (torch.float16, 300, 49153, 3),
                                           (torch.float32, 300, 30011, 0), (torch.bfloat16, 300, 150001, 0), (torch.bfloat16, 600, 35001, 0), (torch.float32, 543, 117813, 0), (torch.float16, 200, 113000, 0), (torch.float16, 3000, 513, 1)])
def test_policy_many_rows(dtype, m, v, pad):
    x = make(m, v, dtype, v, pad)
    x["index"][3] = -1
    x["index"][5] = v - 1
    x["index"][6] = 0
    x["logits"][9, 5:] = torch.finfo(dtype).min
    x["index"][9] = 2
    x["logits"][11, 1:] = -math.inf
    x["index"][11] = 0
    loss, logp, stats, d = check_policy(x)
    form = {"old_logp": x["old"], "ref_logp": x["ref"], "kl": 0.05, "clip_low": LOW, "clip_high": HIGH}
    for _ in range(20):
        again = bz.policy(x["logits"], x["index"], x["adv"], **form, dloss=x["dloss"])
        assert torch.equal(again[0], loss) and torch.equal(again[2].view(torch.int32), stats.view(torch.int32)) and torch.equal(again[3], d)


@pytest.mark.parametrize("pad,where", [(1, 0), (5, 3), (8, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_policy_rows_that_sit_differently(dtype, pad, where):
    for m in (5, 300):
        x = make(m, 2049, dtype, pad, pad)
        out = torch.full((m, 2100), 7.0, dtype=dtype, device="cuda")
        check_policy(x, dlogits=out[:, where:where + 2049])
        assert (out[:, :where] == 7).all() and (out[:, where + 2049:] == 7).all()


def test_policy_forms():
    """On policy, no KL term, no advantage, an infinite upper border, ratios beyond binary32."""
    x = make(60, 300, torch.float32, 4)
    check_policy(x, on_policy=True)
    check_policy(x, kl=0.0)
    x["adv"][::3] = 0.0
    check_policy(x)
    loss, _, stats = bz.policy(x["logits"], x["index"], x["adv"], old_logp=x["old"], clip_low=1.0, clip_high=math.inf)
    lp, _, there, _ = tokens(x["logits"], x["index"], 1.0)
    want = torch.where(there, -torch.exp(lp - x["old"].cpu().double()) * x["adv"].cpu().double(), torch.zeros_like(lp))
    assert near(loss, want, 2 * TOL * want.abs()) and near(stats[:, 2], want, 2 * TOL * want.abs())
    x["old"] -= 500.0        # r beyond every border: clipped where A > 0, without slope there
    loss, _, stats = bz.policy(x["logits"], x["index"], x["adv"], old_logp=x["old"], clip_low=LOW, clip_high=HIGH)
    up = (x["adv"] > 0) & (x["index"] >= 0)
    assert torch.allclose(loss[up], -x["adv"][up] * (1 + HIGH)) and (stats[up][:, 2] == 0).all()
    none = x["adv"] == 0
    assert (loss[none] == 0).all() and (stats[none][:, 2] == 0).all()
    assert (loss[(x["adv"] < 0) & (x["index"] >= 0)] == math.inf).all()


@pytest.mark.parametrize("m", [8, 400])
def test_rows_without_a_token(m):
    """They count for nothing, whatever their logits; tokens out of range have none; tokens of no probability take no gradient."""
    x = make(m, 5000, torch.bfloat16, 2)
    x["index"] = torch.arange(m, dtype=torch.int32, device="cuda") * 7 % 5000
    x["index"][0], x["index"][1], x["index"][2] = -1, 5000, 2 ** 31 - 1
    x["logits"][0] = math.nan
    x["logits"][1] = math.inf
    x["logits"][2] = -math.inf
    x["logits"][3] = -math.inf                     # nothing left of the row
    x["logits"][4, int(x["index"][4])] = -math.inf
    x["logits"][5, 100:] = -math.inf
    loss, logp, stats, d = bz.policy(x["logits"], x["index"], x["adv"], old_logp=x["old"], ref_logp=x["ref"], kl=0.1, dloss=x["dloss"])
    assert (loss[:3] == 0).all() and (logp[:3] == 0).all() and (d[:5] == 0).all() and (stats[:5, 2] == 0).all()
    assert (logp[3:5] == -math.inf).all() and (loss[3:5] == math.inf).all()
    assert torch.isfinite(d).all() and torch.isfinite(logp[5:]).all() and (d[5, 100:] == 0).all()
    x["logits"][6, 17] = math.nan
    _, logp, _, d = bz.policy(x["logits"], x["index"], x["adv"], dloss=x["dloss"])
    assert logp[6].isnan() and d[6].isnan().all() and torch.isfinite(d[7:]).all()


def preference_reference(x, starts, pairs, T, beta, margin, smoothing, mean, dloss):
    m = x["logits"].shape[0]
    lp, q, there, at = tokens(x["logits"], x["index"], T)
    ref = x["ref"].cpu().double() if x["ref"] is not None else torch.zeros(m, dtype=torch.float64)
    clamp = [min(max(int(s), 0), m) for s in starts]
    reward, share, rows = torch.zeros(2 * pairs, dtype=torch.float64), torch.zeros(2 * pairs, dtype=torch.float64), []
    wobble = torch.zeros(2 * pairs, dtype=torch.float64)
    for n in range(2 * pairs):
        part = [i for i in range(clamp[n], clamp[n + 1]) if there[i]]
        rows.append((clamp[n], clamp[n + 1]))
        share[n] = beta / (max(len(part), 1) if mean else 1)
        reward[n] = share[n] * sum(float(lp[i] - ref[i]) for i in part)
        wobble[n] = abs(share[n]) * TOL * len(part) + F32 * abs(reward[n])
    h = reward[:pairs] - reward[pairs:] - margin
    soft = torch.nn.functional.softplus
    loss = (1 - smoothing) * soft(-h) + smoothing * soft(h)
    dh = smoothing * torch.sigmoid(h) - (1 - smoothing) * torch.sigmoid(-h)
    slope, bend, up = torch.zeros(m, dtype=torch.float64), torch.zeros(m, dtype=torch.float64), torch.zeros(m, dtype=torch.float64)
    for n, (a, b) in enumerate(rows):
        p = n % pairs
        slope[a:b] = (dh[p] if n < pairs else -dh[p]) * share[n]
        up[a:b] = dloss[p]
        # how far the pair's wobble moves the slope, in units of TOL
        bend[a:b] = abs(share[n]) * 0.25 * (wobble[p] + wobble[p + pairs]) / TOL
    slope = torch.where(lp == -math.inf, torch.zeros_like(slope), slope)
    d, bound = gradient(q, there, at, slope, bend, up, T)
    return loss, reward, lp, d, bound, wobble[:pairs] + wobble[pairs:], wobble


def check_preference(x, starts, T=1.0, beta=0.1, margin=0.0, smoothing=0.0, mean=False, dlogits=None):
    pairs = len(starts) // 2
    dloss = x["dloss"][:pairs].contiguous()
    form = {"ref_logp": x["ref"], "beta": beta, "margin": margin, "smoothing": smoothing, "mean": mean, "temperature": T}
    s = torch.tensor(starts, dtype=torch.int32, device="cuda")
    want, reward, lp, wd, bound, wobble, each = preference_reference(x, starts, pairs, T, beta, margin, smoothing, mean, dloss.cpu().double())
    got = bz.preference(x["logits"], x["index"], s, **form, dloss=dloss, dlogits=dlogits)
    d = got[4]
    bound = bound + HALF_UNIT[d.dtype] * wd.abs() + TINY[d.dtype]
    assert near(got[0], want, wobble + 2 * F32 * want.abs()) and near(got[1], reward, each) and near(got[2], lp, TOL + F32 * lp.abs())
    assert near(d, wd, bound)
    only = bz.preference(x["logits"], x["index"], s, **form)
    assert len(only) == 4 and all(torch.equal(a, b) for a, b in zip(only[:3], got[:3]))
    assert torch.equal(bz.token_loss_backward(x["logits"], x["index"], only[3], dloss, T, dlogits=torch.empty_like(d)), d) or dlogits is not None
    return got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v,starts", [(2, 3, [0, 1, 2]), (10, 100, [0, 4, 10]), (9, 1001, [1, 1, 3, 8, 8]), (40, 333, [0, 5, 9, 20, 22, 22, 36]), (6, 70001, [0, 2, 6]),
                                        (300, 9000, [0, 10, 100, 150, 290]), (400, 5003, [3, 70, 180, 181, 399])])
def test_preference_matches(m, v, starts, dtype):
    x = make(m, v, dtype, v)
    check_preference(x, starts)
    check_preference(x, starts, T=1.5, beta=0.3, margin=0.2, smoothing=0.1, mean=True)


@pytest.mark.parametrize("pad,where", [(1, 0), (5, 3)])
def test_preference_other_forms(pad, where):
    x = make(50, 515, torch.float16, pad, pad)
    out = torch.full((50, 600), 7.0, dtype=torch.float16, device="cuda")
    check_preference(x, [0, 20, 44], dlogits=out[:, where:where + 515])
    assert (out[:, :where] == 7).all() and (out[:, where + 515:] == 7).all() and (out[44:, where:where + 515] == 0).all()
    x["ref"] = None
    check_preference(x, [0, 20, 44], smoothing=1.0)
    check_preference(x, [-5, 20, 10 ** 6])                          # taken into [0, m]
    x["index"][:] = -1
    loss, reward, logp, stats, d = check_preference(x, [0, 20, 44], mean=True, margin=1.0)
    assert (reward == 0).all() and (d == 0).all() and torch.allclose(loss.cpu().double(), torch.nn.functional.softplus(torch.tensor([1.0], dtype=torch.float64)))


def test_preference_far_apart():
    """h of hundreds: one side's loss is h itself, the other's vanishes, and the slopes keep their digits."""
    x = make(40, 200, torch.float32, 1)
    check_preference(x, [0, 10, 20, 30, 40], beta=20.0)
    check_preference(x, [0, 10, 20, 30, 40], beta=-20.0, smoothing=0.2)


@pytest.mark.parametrize("low, peak", [(-math.inf, 0.0), (torch.finfo(torch.float32).min, 0.0), (torch.finfo(torch.float32).min, 1e38)])
def test_preference_with_tokens_of_no_probability(low, peak):
    """A chosen token whose logit is -inf, or whose logarithm is as low as binary32 goes or, counted as -inf, lower: reward and loss are the
    formula's rounded to binary32 (half the lowest value where the logarithm still is one), the other rows' slopes those of a lost pair, and
    the token takes a gradient where its logarithm is finite."""
    x = make(8, 40, torch.float32, 2)
    x["index"] = torch.arange(8, dtype=torch.int32, device="cuda")
    x["logits"][1, 1] = low
    x["logits"][1, 2] += peak
    loss, reward, logp, _, d = bz.preference(x["logits"], x["index"], torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"), ref_logp=x["ref"], beta=0.5,
                                             dloss=torch.ones(1, device="cuda"))
    lp = torch.log_softmax(x["logits"].double(), 1)[torch.arange(8), torch.arange(8)]
    lp[1] = float(lp[1].float())
    assert float(logp[1]) == float(lp[1])
    chosen, rejected = (0.5 * (lp - x["ref"].double())).view(2, 4).sum(1)
    assert float(reward[0]) == float(chosen.float()) and torch.isfinite(reward[1]) and float(loss) == float((rejected - chosen).float())
    p = torch.softmax(x["logits"].double(), 1)
    want = -0.5 * (torch.eye(8, 40, dtype=torch.float64, device="cuda") - p)
    want[4:] *= -1
    if float(lp[1]) == -math.inf:
        want[1] = 0
    assert (d.double() - want).abs().max() < 1e-6


@pytest.mark.parametrize("dtype,m,v,pad", [(torch.bfloat16, 300, 4100, 0), (torch.bfloat16, 300, 5113, 0), (torch.float32, 300, 2551, 1), (torch.bfloat16, 200, 40001, 0),
                                           (torch.float16, 160, 50257, 0), (torch.float16, 160, 65537, 5), (torch.float32, 100, 65531, 0), (torch.bfloat16, 100, 160001, 0)])
def test_policy_lengths_between_batches(dtype, m, v, pad):
    """Rows whose words leave a CTA, or the last of a row's, batches that are not full: one warp's, and those of three to eight CTAs."""
    x = make(m, v, dtype, v, pad)
    x["index"][:4] = torch.tensor([0, v - 1, -1, v], dtype=torch.int32)
    check_policy(x, 1.0, 0.05)


def test_gradient_of_losses_that_dloss_does_not_hold():
    """Stats of one loss with an upstream gradient of another length: rows whose place it has not get NaN, rows without a slope 0."""
    for dtype in DTYPES:
        x = make(12, 70, dtype, 3)
        x["index"] = torch.arange(12, dtype=torch.int32, device="cuda")
        x["index"][[2, 9]] = -1
        _, _, stats, want = bz.policy(x["logits"], x["index"], x["adv"], clip_low=1.0, clip_high=math.inf, dloss=x["dloss"])
        got = bz.token_loss_backward(x["logits"], x["index"], stats, x["dloss"][:5].clone())
        want, size = want[:5].cpu().double(), (x["adv"] * x["dloss"])[:5, None].cpu().double().abs()
        # two computations of slope times (indicator less softmax), each within 3 TOL of its terms, and their roundings
        assert near(got[:5], want, 2 * (3 * TOL * 2 * size + HALF_UNIT[dtype] * (want.abs() + 6 * TOL * size) + TINY[dtype]))
        assert got[9].eq(0).all() and got[[5, 6, 7, 8, 10, 11]].isnan().all()
        assert bz.token_loss_backward(x["logits"], x["index"], stats, x["dloss"][:0].clone())[[0, 11]].isnan().all()
        stats = bz.preference(x["logits"], x["index"], torch.tensor([0, 3, 6, 9, 12], dtype=torch.int32, device="cuda"), dloss=x["dloss"][:2].clone())[3]
        got = bz.token_loss_backward(x["logits"], x["index"], stats, x["dloss"][:1].clone())
        assert got[[2, 9]].eq(0).all() and got[[3, 4, 5, 10, 11]].isnan().all() and got[[0, 1, 6, 7, 8]].isfinite().all()


def test_preference_many_pairs():
    m, pairs = 4000, 1000
    x = make(m, 50, torch.bfloat16, 3)
    x["dloss"] = torch.rand(pairs, device="cuda") + 0.5
    check_preference(x, [2 * k for k in range(2 * pairs + 1)])


@pytest.mark.parametrize("v,m", [(1000, 6), (50000, 6), (300001, 6), (20000, 300), (9, 6)])
def test_in_place_other_stream_graph_and_same_bits(v, m):
    x = make(m, v, torch.bfloat16, 1)
    starts = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    pair_loss = torch.ones(1, device="cuda")
    form = {"old_logp": x["old"], "ref_logp": x["ref"], "kl": 0.1}
    want = bz.policy(x["logits"], x["index"], x["adv"], **form, dloss=x["dloss"])
    want2 = bz.preference(x["logits"], x["index"], starts, ref_logp=x["ref"], dloss=pair_loss)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a, b, c = x["logits"].clone(), x["logits"].clone(), x["logits"].clone()
        bz.policy(a, x["index"], x["adv"], **form, dloss=x["dloss"], dlogits=a)
        bz.preference(b, x["index"], starts, ref_logp=x["ref"], dloss=pair_loss, dlogits=b)
        bz.token_loss_backward(c, x["index"], want2[3], pair_loss, dlogits=c)
    s.synchronize()
    assert torch.equal(a, want[3]) and torch.equal(b, want2[4]) and torch.equal(c, want2[4])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = bz.policy(x["logits"], x["index"], x["adv"], **form, dloss=x["dloss"])
        got2 = bz.preference(x["logits"], x["index"], starts, ref_logp=x["ref"], dloss=pair_loss)
    for _ in range(3):
        graph.replay()
    assert all(torch.equal(p, q) for p, q in zip((got[0], got[1], got[3], *got2[:3], got2[4]), (want[0], want[1], want[3], *want2[:3], want2[4])))
    x["logits"].neg_()
    graph.replay()
    assert torch.equal(got[3], bz.policy(x["logits"], x["index"], x["adv"], **form, dloss=x["dloss"])[3])


def test_gradients_against_differences():
    x = make(4, 12, torch.float32, 5)
    x["index"] = torch.tensor([3, 0, 11, 7], dtype=torch.int32, device="cuda")
    lp = tokens(x["logits"], x["index"], 2.0)[0]
    x["old"] = (lp - torch.tensor([0.1, -0.1, 0.05, 0.0])).float().cuda()
    form = {"old_logp": x["old"], "ref_logp": x["ref"], "kl": 0.3, "clip_low": LOW, "clip_high": HIGH, "temperature": 2.0}
    d = bz.policy(x["logits"], x["index"], x["adv"], **form, dloss=x["dloss"])[3]
    starts = [0, 2, 4]
    e = bz.preference(x["logits"], x["index"], torch.tensor(starts, dtype=torch.int32, device="cuda"), ref_logp=x["ref"], beta=0.7, smoothing=0.1, dloss=x["dloss"][:1].contiguous())[4]
    step = 1e-4
    for i, c in [(0, 0), (0, 3), (1, 0), (2, 11), (3, 5)]:
        policy, pref = [], []
        for sign in (1, -1):
            y = dict(x, logits=x["logits"].cpu().double())
            y["logits"][i, c] += sign * step
            lp = tokens(y["logits"], y["index"], 2.0)[0]
            policy.append(policy_reference(lp, x["old"].cpu().double(), x["ref"].cpu().double(), x["adv"].cpu().double(), 0.3)[0][i])
            pref.append(preference_reference(y, starts, 1, 1.0, 0.7, 0.0, 0.1, False, x["dloss"].cpu().double())[0][0])
        assert abs(float(policy[0] - policy[1]) / (2 * step) * float(x["dloss"][i]) - float(d[i, c])) < 5e-6
        assert abs(float(pref[0] - pref[1]) / (2 * step) * float(x["dloss"][0]) - float(e[i, c])) < 5e-6


def test_no_vocabulary_and_no_positions():
    index = torch.zeros(3, dtype=torch.int32, device="cuda")
    some = torch.ones(3, device="cuda")
    for x in bz.policy(torch.empty(3, 0, device="cuda"), index, some)[:2]:
        assert (x == 0).all()
    starts = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")
    loss, reward, logp, stats = bz.preference(torch.empty(3, 0, device="cuda"), index, starts)
    assert (logp == 0).all() and (reward == 0).all() and torch.allclose(loss, torch.full_like(loss, math.log(2.0)))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert bz.policy(torch.empty(0, 9, device="cuda"), none, torch.empty(0, device="cuda"))[0].numel() == 0
    loss, reward, _, _ = bz.preference(torch.empty(0, 9, device="cuda"), none, starts)
    assert (reward == 0).all() and torch.allclose(loss, torch.full_like(loss, math.log(2.0)))
    x = make(4, 30, torch.float32, 0)
    loss, reward, logp, stats, d = bz.preference(x["logits"], x["index"], torch.zeros(1, dtype=torch.int32, device="cuda"), dloss=torch.empty(0, device="cuda"))
    assert loss.numel() == 0 and (d == 0).all() and near(logp, tokens(x["logits"], x["index"], 1.0)[0], 2 * TOL)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,v", [(9, 500), (400, 9001), (300, 70001)])
def test_rows_far_from_zero(dtype, m, v):
    """Rows of the type's lowest value alone (every token is as likely), lowest values beside ordinary ones, logits around a large number."""
    x = make(m, v, dtype, 11)
    low = torch.finfo(dtype).min
    x["index"] = torch.full((m,), 3, dtype=torch.int32, device="cuda")
    x["logits"][0] = low
    x["logits"][1] = low
    x["logits"][1, 3] = 1.0
    x["logits"][2, ::2] = low
    x["logits"][3] = 30000.0
    x["logits"][3, 3] += 32.0
    x["logits"][4] = -30000.0
    loss, logp, stats, d = bz.policy(x["logits"], x["index"], torch.ones(m, device="cuda"), dloss=torch.ones(m, device="cuda"))
    lp, q, there, at = tokens(x["logits"][:6], x["index"][:6], 1.0)
    assert near(logp[:6], lp, TOL + F32 * lp.abs())
    want, bound = gradient(q, there, at, -torch.ones(6, dtype=torch.float64), torch.ones(6, dtype=torch.float64), torch.ones(6, dtype=torch.float64), 1.0)
    assert near(d[:6], want, bound + HALF_UNIT[dtype] * want.abs() + TINY[dtype])
    assert near(bz.token_loss_backward(x["logits"], x["index"], stats)[:6], want, bound + HALF_UNIT[dtype] * want.abs() + TINY[dtype])


def test_two_threads_with_different_sizes():
    """Each call's launch is its own: rows of 70 KB of shared memory beside short ones, from two host threads on two streams."""
    import threading
    jobs = [make(300, 35001, torch.bfloat16, 1), make(300, 900, torch.bfloat16, 2)]
    want = [bz.policy(x["logits"], x["index"], x["adv"], dloss=x["dloss"])[3] for x in jobs]
    torch.cuda.synchronize()
    failed = []

    def run(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(100):
                    got = bz.policy(jobs[k]["logits"], jobs[k]["index"], jobs[k]["adv"], dloss=jobs[k]["dloss"])[3]
                torch.cuda.current_stream().synchronize()
                failed.append(not torch.equal(got, want[k]))
        except Exception as e:      # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=run, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert failed == [False, False]
