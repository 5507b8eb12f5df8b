"""bz_distill and bz_distill_backward against the formula in 64 bits.

Tolerances.  With logits of size below 40 at temperature 1 the exponent's argument is known to about
40 * 1.44 * 2^-23 = 7e-6, so q and p are within 1e-5 relative; dlogits = dloss*T*(q - p) then within
1e-5 * |dloss| T (q + p) plus half a unit of its type; the loss is a p-weighted mean of differences of logarithms,
each known to about 1e-5, times T^2.
"""
import math

import pytest
import torch

from paper_2010_04902_b200 import binding as bz

pytestmark = pytest.mark.gpu

HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}
TOL = 1e-5


def reference(logits, teacher, index, T, dloss):
    m, v = logits.shape
    s = logits.detach().cpu().double() / T
    loss, d, size = torch.zeros(m, dtype=torch.float64), torch.zeros(m, v, dtype=torch.float64), torch.zeros(m, v, dtype=torch.float64)
    lse = torch.logsumexp(s, 1)
    for i in range(m):
        kept = [(int(c), float(z) / T) for c, z in zip(index[i], teacher[i]) if 0 <= int(c) < v and float(z) != -math.inf]
        if not kept:
            continue
        z = torch.tensor([k[1] for k in kept], dtype=torch.float64)
        log_p = z - torch.logsumexp(z, 0)
        log_q = s[i] - lse[i] if lse[i] > -math.inf else torch.full((v,), -math.inf, dtype=torch.float64)
        q = torch.exp(log_q)
        d[i] += q
        size[i] += q
        for (c, _), lp in zip(kept, log_p):
            p = math.exp(lp)
            if p > 0:
                loss[i] += p * (lp - log_q[c])
            d[i, c] -= p
            size[i, c] += p
        d[i] *= float(dloss[i]) * T
        size[i] *= abs(float(dloss[i])) * T
    return T * T * loss, lse, d, size


def make(m, v, t, dtype, seed, pad=0, gone=True):
    g = torch.Generator().manual_seed(seed)
    logits = (torch.randn(m, v + pad, generator=g) * 2.5).to(dtype)[:, :v]
    teacher = torch.randn(m, t, generator=g) * 3
    index = torch.randint(0, v, (m, t), generator=g, dtype=torch.int32)   # repeats happen, and more often in small v
    if gone:
        u = torch.rand(m, 1, generator=g)
        index = torch.where((u < 0.3) & (torch.arange(t)[None] >= t // 2), torch.full_like(index, -1), index)
    dloss = torch.rand(m, generator=g) + 0.5
    full = torch.empty(m, v + pad, dtype=dtype, device="cuda")
    full[:, :v] = logits.cuda()
    return full[:, :v], teacher.cuda(), index.cuda().contiguous(), dloss.cuda()


def check(logits, teacher, index, T, dloss, dlogits=None):
    want_loss, want_lse, want_d, size = reference(logits, teacher, index, T, dloss)
    loss, stats, d = bz.distill(logits, teacher, index, T, dloss=dloss, dlogits=dlogits)
    near = lambda got, want, tol: bool(((got.cpu().double() == want) | ((got.cpu().double() - want).abs() <= tol)).all())  # noqa: E731
    assert near(loss, want_loss, TOL * T * T + TOL * want_loss.abs())
    lse = stats[:, 0].double() / T + torch.log(stats[:, 1].double())
    assert near(lse, want_lse, TOL)
    bound = 2 * TOL * size + HALF_UNIT[d.dtype] * want_d.abs() + TINY[d.dtype]
    assert near(d, want_d, bound)
    only, stats2 = bz.distill(logits, teacher, index, T)
    assert near(only, want_loss, TOL * T * T + TOL * want_loss.abs())
    if dlogits is None:    # rows that sit alike: the same order of sums
        assert torch.equal(only, loss) and torch.equal(stats2, stats)
    assert near(bz.distill_backward(logits, teacher, index, stats, dloss, T), want_d, bound)
    return loss, lse, d


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,v,t,T", [(1, 1, 1, 1.0), (3, 2, 5, 2.0), (5, 33, 1, 1.0), (4, 500, 7, 0.5), (7, 1001, 64, 4.0), (3, 1024, 128, 1.0),
                                     (2, 8193, 33, 2.0), (2, 32768, 50, 1.0), (2, 32771, 50, 1.0), (3, 70001, 16, 2.0), (2, 200003, 9, 1.0),
                                     (1, 300001, 12, 1.0)])
def test_matches(m, v, t, T, dtype):
    check(*make(m, v, t, dtype, seed=v + t)[:3], T, make(m, v, t, dtype, seed=v + t)[3])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_padding_entries_never_leave_their_row(dtype):
    """Entries without an index next to rows that begin off a 16-byte boundary: every other row of an odd length."""
    logits, teacher, index, dloss = make(16, 1003, 8, dtype, seed=3)
    index[::2, 3:] = -1
    index[5] = -1
    check(logits, teacher, index, 1.0, dloss)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("pad,where", [(1, 0), (5, 3), (8, 0)])
def test_rows_that_sit_differently(dtype, pad, where):
    logits, teacher, index, dloss = make(5, 2049, 20, dtype, seed=pad, pad=pad)
    out = torch.full((5, 2100), 7.0, dtype=dtype, device="cuda")
    check(logits, teacher, index, 2.0, dloss, dlogits=out[:, where:where + 2049])
    assert (out[:, :where] == 7).all() and (out[:, where + 2049:] == 7).all()


def test_entries_that_do_not_count():
    m, v = 8, 100
    logits, teacher, index, dloss = make(m, v, 6, torch.float32, seed=1, gone=False)
    index[0] = -1                           # a padded position
    index[1] = v                            # out of range: not kept either
    index[2, 1:] = 2 ** 31 - 1
    teacher[3] = -math.inf                  # indices but no weight
    teacher[4, 2:] = -math.inf
    index[5] = 7                            # one place, six entries
    loss, lse, d = check(logits, teacher, index, 1.0, dloss)
    for i in (0, 1, 3):
        assert float(loss[i]) == 0 and (d[i] == 0).all()
    assert abs(float(d[5].sum())) < 1e-5


def test_masked_vocabulary():
    logits, teacher, index, dloss = make(4, 300, 5, torch.float16, seed=2, gone=False)
    logits[0, 100:] = -math.inf
    index[0] = torch.arange(5)
    logits[1] = -math.inf                   # nothing left of the student
    logits[2, 10] = -math.inf
    index[2, 0] = 10                        # the teacher wants what the student cannot give
    logits[3] = -1000.0
    logits[3, ::3] = -math.inf
    index[3] = torch.tensor([1, 2, 4, 5, 7])
    loss, lse, d = check(logits, teacher, index, 1.0, dloss)
    assert float(loss[1]) == math.inf and float(loss[2]) == math.inf and math.isfinite(float(loss[0])) and math.isfinite(float(loss[3]))
    assert torch.isfinite(d).all() and float(lse[1]) == -math.inf


@pytest.mark.parametrize("v", [1000, 50000, 300001])
def test_in_place_other_stream_and_same_bits(v):
    logits, teacher, index, dloss = make(6, v, 40, torch.bfloat16, seed=1)
    loss, stats, d = bz.distill(logits, teacher, index, 2.0, dloss=dloss)
    for _ in range(10):
        loss2, _, d2 = bz.distill(logits, teacher, index, 2.0, dloss=dloss)
        assert torch.equal(loss, loss2) and torch.equal(d, d2)
    alone = bz.distill_backward(logits, teacher, index, stats, dloss, 2.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a, b = logits.clone(), logits.clone()
        bz.distill(a, teacher, index, 2.0, dloss=dloss, dlogits=a)
        bz.distill_backward(b, teacher, index, stats, dloss, 2.0, dlogits=b)
    s.synchronize()
    assert torch.equal(a, d) and torch.equal(b, alone)


def test_gradient_against_differences():
    logits, teacher, index, dloss = make(2, 12, 4, torch.float32, seed=5, gone=False)
    _, _, d = bz.distill(logits, teacher, index, 2.0, dloss=dloss)
    step = 1e-4
    for i, c in [(0, 0), (0, int(index[0, 0])), (1, 3), (1, int(index[1, 2]))]:
        up, down = logits.cpu().double(), logits.cpu().double()
        up[i, c] += step
        down[i, c] -= step
        diff = (reference(up, teacher, index, 2.0, dloss)[0][i] - reference(down, teacher, index, 2.0, dloss)[0][i]) / (2 * step)
        assert abs(float(diff) * float(dloss[i]) - float(d[i, c])) < 5e-6


@pytest.mark.parametrize("dtype,v,pad,t", [(torch.bfloat16, 8200, 0, 5), (torch.bfloat16, 8201, 0, 40), (torch.float32, 4111, 1, 3), (torch.float16, 49140, 0, 33),
                                           (torch.float16, 49153, 3, 64), (torch.float32, 30011, 0, 300), (torch.bfloat16, 150001, 0, 8)])
def test_many_rows(dtype, v, pad, t):
    """Rows enough for the ring: shorter than one chunk, several chunks, longer than what is held."""
    m = 300 if v > 100000 else 500
    logits, teacher, index, dloss = make(m, v, t, dtype, seed=v + t, pad=pad)
    index[3] = -1
    index[m - 1, 1:] = index[m - 1, 0]
    logits[7] = -math.inf
    logits[9, 5:] = torch.finfo(dtype).min
    some = [0, 1, 2, 3, 7, 9, 147, 148, 149, 295, 296, 297, m - 2, m - 1]
    out = torch.empty_like(logits) if pad == 0 else torch.empty(m, v + pad, dtype=dtype, device="cuda")[:, :v]
    loss, stats, d = bz.distill(logits, teacher, index, 2.0, dloss=dloss, dlogits=out)
    want_loss, want_lse, want_d, size = reference(logits[some], teacher[some], index[some], 2.0, dloss[some])
    want_loss = want_loss.float().double()    # row 9's is beyond binary32: an infinity there
    near = lambda got, want, tol: bool(((got.cpu().double() == want) | ((got.cpu().double() - want).abs() <= tol)).all())  # noqa: E731
    assert near(loss[some], want_loss, 4 * TOL + TOL * want_loss.abs())
    assert near(d[some], want_d, 2 * TOL * size + HALF_UNIT[dtype] * want_d.abs() + TINY[dtype])
    # every row against the two other kernels: a few rows at a time, and the gradient alone
    for lo in range(0, m, 100):
        part = slice(lo, lo + 100)
        few, few_stats, few_d = bz.distill(logits[part], teacher[part].contiguous(), index[part].contiguous(), 2.0, dloss=dloss[part].contiguous())
        assert near(loss[part], few.cpu().double(), 8 * TOL + 2 * TOL * few.cpu().double().abs().clamp(max=1e30))
        same = (d[part].float() - few_d.float()).abs() <= (2 * HALF_UNIT[dtype] + 4 * TOL) * few_d.float().abs() + 4 * TOL * dloss[part][:, None] + TINY[dtype]
        assert same.all() and torch.equal(stats[part][:, 0], few_stats[:, 0])
        assert torch.allclose(stats[part][:, 1], few_stats[:, 1], rtol=TOL)
    for _ in range(30):
        loss2, stats2, d2 = bz.distill(logits, teacher, index, 2.0, dloss=dloss, dlogits=torch.empty_like(logits) if pad == 0 else torch.empty(m, v + pad, dtype=dtype, device="cuda")[:, :v])
        assert torch.equal(loss, loss2) and torch.equal(stats, stats2) and torch.equal(d, d2)
    only, stats2 = bz.distill(logits, teacher, index, 2.0)
    assert torch.equal(only, loss) and torch.equal(stats2, stats)
    if pad == 0:
        bz.distill(logits, teacher, index, 2.0, dloss=dloss, dlogits=logits)
        assert torch.equal(logits, d)


def test_many_entries():
    logits, teacher, index, dloss = make(2, 5000, 1024, torch.float32, seed=5)
    check(logits, teacher, index, 1.0, dloss)


def test_no_vocabulary_and_no_positions():
    loss, stats = bz.distill(torch.empty(3, 0, device="cuda"), torch.zeros(3, 2, device="cuda"),
                           torch.zeros(3, 2, dtype=torch.int32, device="cuda"))
    assert (loss == 0).all() and (stats[:, 0] == -math.inf).all() and (stats[:, 1] == 0).all()
    loss, _ = bz.distill(torch.empty(0, 9, device="cuda"), torch.zeros(0, 2, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    assert loss.numel() == 0


@pytest.mark.parametrize("dtype,v,grad", [(torch.float16, 50003, False), (torch.bfloat16, 32128, False), (torch.bfloat16, 40000, True), (torch.float32, 9001, True)])
def test_ring_gives_the_same_bits_over_many_calls(dtype, v, grad):
    """Rows enough to go round the ring several times a CTA, read once and read twice."""
    logits, teacher, index, dloss = make(900, v, 16, dtype, seed=v)
    how = {"dloss": dloss, "dlogits": torch.empty_like(logits)} if grad else {}
    loss, stats = (t.clone() for t in bz.distill(logits, teacher, index, 2.0, **how)[:2])
    differs = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(500):
        again = bz.distill(logits, teacher, index, 2.0, **how)
        differs += (again[0] != loss).any() | (again[1] != stats).any()
    assert int(differs) == 0


@pytest.mark.parametrize("T", [5e-39, 1e-30, 1e-3])
def test_smallest_temperatures(T):
    """q is all on the largest logit; the teacher names it alone, or another one."""
    logits = torch.randn(2, 50, generator=torch.Generator().manual_seed(1)).cuda()
    top = logits.argmax(1).to(torch.int32)
    loss, _, d = bz.distill(logits, torch.zeros(2, 1, device="cuda"), top[:, None].contiguous(), T, dloss=torch.ones(2, device="cuda"))
    assert (loss == 0).all() and (d == 0).all()
    other = ((top + 1) % 50).to(torch.int32)
    _, _, d = bz.distill(logits, torch.zeros(2, 1, device="cuda"), other[:, None].contiguous(), T, dloss=torch.ones(2, device="cuda"))
    want = torch.zeros(2, 50)     # set on the host: an addition on the GPU by atomics would flush the smallest T
    for i in range(2):
        want[i, int(top[i])], want[i, int(other[i])] = T, -T
    assert torch.equal(d.cpu(), want)
