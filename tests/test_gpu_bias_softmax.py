"""bz_bias_softmax and its gradient against the formulas in 64 bits: types, odd lengths, strides, masks that leave
rows empty, values at the ends of the types' ranges, and repeated launches that have to agree bit for bit.

Tolerances.  A result is rounded once to its type (half a unit in the last place: 2^-24, 2^-11, 2^-8 relative for
binary32, binary16, bfloat16).  Before that, binary32 arithmetic: the exponent's argument (z - max)*log2(e) is
known to about 2^-23 of its terms' size (|z| here stays below 40, so 40 * 1.44 * 2^-23 = 7e-6 relative in p),
2^x and the sums add a few units of 2^-23.  So p is within 1e-5 relative plus its type's half unit, dz = p (dp - D)
within that times |p| (|dp| + |D|), and a table gradient within 1e-5 of the sum of its terms' sizes.
"""
import math

import pytest
import torch

from paper_2010_04902_b200 import binding as bz

pytestmark = pytest.mark.gpu

HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}  # below: subnormal or flushed
P_TOL = 1e-5


def bucket(rel, buckets, distance, both):
    """The rule of the header, one integer at a time."""
    nb = buckets // 2 if both else buckets
    n = abs(rel) if both else max(-rel, 0)
    e = nb // 2
    if n < e:
        c = n
    else:
        steps = nb - e
        c = e + max(t for t in range(steps) if n ** steps >= e ** (steps - t) * distance ** t)
    return c + nb if both and rel > 0 else c


def reference(scores, table, distance, both, causal, scale, k_len, q_start, dprobs=None):
    b, h, tq, tk = scores.shape
    p_all = torch.zeros(scores.shape, dtype=torch.float64)
    lse_all = torch.full((b, h, tq), -math.inf, dtype=torch.float64)
    ds_all = torch.zeros(scores.shape, dtype=torch.float64)
    size_all = torch.zeros(scores.shape, dtype=torch.float64)
    dt = torch.zeros(table.shape, dtype=torch.float64)
    dt_size = torch.zeros(table.shape, dtype=torch.float64)
    s64, t64 = scores.detach().cpu().double(), table.detach().cpu().double()
    lut = {}
    for ib in range(b):
        keys = tk if k_len is None else max(0, min(tk, int(k_len[ib])))
        start = 0 if q_start is None else int(q_start[ib])
        for i in range(tq):
            end = min(keys, max(0, i + start + 1)) if causal else keys
            if end == 0:
                continue
            kinds = torch.tensor([lut.setdefault(r, bucket(r, table.shape[0], distance, both)) for r in range(-i - start, end - i - start)])
            z = scale * s64[ib, :, i, :end] + t64[kinds].T
            lse = torch.logsumexp(z, -1)
            p = torch.where(torch.isinf(lse)[:, None], torch.zeros_like(z), torch.exp(z - lse[:, None]))
            p_all[ib, :, i, :end] = p
            lse_all[ib, :, i] = lse
            if dprobs is not None:
                dp = dprobs[ib, :, i, :end].detach().cpu().double()
                D = (p * dp).sum(-1, keepdim=True)
                dz = p * (dp - D)
                ds_all[ib, :, i, :end] = scale * dz
                size = p * (dp.abs() + (p * dp.abs()).sum(-1, keepdim=True))
                size_all[ib, :, i, :end] = abs(scale) * size
                dt.index_add_(0, kinds, dz.T)
                dt_size.index_add_(0, kinds, size.T)
    return p_all, lse_all, ds_all, size_all, dt, dt_size


def log_sum(stats):
    return stats[..., 0].cpu().double() + torch.log(stats[..., 1].cpu().double())


def make(b, h, tq, tk, dtype, seed, pad=0, sigma=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(b, h, tq, tk + pad, generator=g) * sigma).to(dtype).cuda()[..., :tk]


def check_forward(scores, table, distance, both, causal=False, scale=1.0, k_len=None, q_start=None, probs=None):
    dev = lambda t: None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    p, stats = bz.bias_softmax(scores, table, distance, both, causal, scale, dev(k_len), dev(q_start), probs=probs)
    want, want_lse, *_ = reference(scores, table, distance, both, causal, scale, k_len, q_start)
    got = p.cpu().double()
    assert ((got - want).abs() <= want * (P_TOL + HALF_UNIT[scores.dtype]) + TINY[scores.dtype]).all()
    none = torch.isinf(want_lse)
    assert (log_sum(stats)[none] == -math.inf).all() and (got[none] == 0).all()
    assert ((log_sum(stats) - want_lse)[~none].abs() <= 1e-5).all()
    return p, stats


def check_backward(scores, table, distance, both, causal=False, scale=1.0, k_len=None, q_start=None, dprobs=None, dscores=None):
    dev = lambda t: None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    _, stats = bz.bias_softmax(scores, table, distance, both, causal, scale, dev(k_len), dev(q_start))
    want = reference(scores, table, distance, both, causal, scale, k_len, q_start, dprobs)
    ds, dt = bz.bias_softmax_backward(scores, table, stats, dprobs, distance, both, causal, scale, dev(k_len), dev(q_start), dscores=dscores)
    _, _, want_ds, size, want_dt, dt_size = want
    got = ds.cpu().double()
    assert ((got - want_ds).abs() <= 2 * P_TOL * size + HALF_UNIT[scores.dtype] * want_ds.abs() + TINY[scores.dtype]).all()
    assert ((dt.cpu().double() - want_dt).abs() <= 2 * P_TOL * dt_size + 1e-30).all()
    return ds, dt


SHAPES = [(1, 1, 1, 1), (2, 3, 5, 7), (1, 2, 33, 64), (3, 2, 17, 255), (1, 2, 9, 256), (1, 2, 9, 257), (2, 1, 20, 1000), (1, 1, 3, 1024),
          (1, 1, 3, 1025), (1, 2, 4, 4096), (1, 1, 3, 4099), (1, 1, 2, 16400)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward_match(shape, dtype):
    b, h, tq, tk = shape
    scores = make(*shape, dtype, seed=tk + tq)
    table = torch.randn(32, h, generator=torch.Generator().manual_seed(tk)).cuda()
    check_forward(scores, table, 128, True)
    check_backward(scores, table, 128, True, dprobs=make(*shape, dtype, seed=1 + tk + tq, sigma=1.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_rows_that_sit_differently(dtype, pad):
    """Scores are a slice, the other tensors are not (or the other way round): the element path."""
    shape = (2, 2, 11, 301)
    scores, dprobs = make(*shape, dtype, seed=5, pad=pad), make(*shape, dtype, seed=6, sigma=1.0)
    table = torch.randn(16, 2, generator=torch.Generator().manual_seed(3)).cuda()
    out = torch.full((2, 2, 11, 320), 7.0, dtype=dtype, device="cuda")
    check_forward(scores, table, 40, True, probs=out[..., 5:306])
    assert (out[..., :5] == 7).all() and (out[..., 306:] == 7).all()
    check_backward(scores, table, 40, True, dprobs=dprobs)
    # heads and queries stored in another order
    swapped = scores.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    check_forward(swapped, table, 40, True)
    check_backward(swapped, table, 40, True, dprobs=dprobs)


@pytest.mark.parametrize("both,buckets,distance", [(True, 4, 2), (True, 32, 128), (True, 64, 200), (False, 2, 2), (False, 3, 9), (False, 32, 128),
                                                   (True, 32, 336), (False, 32, 400), (True, 48, 512), (False, 16, 2048), (True, 256, 2048)])
def test_bucket_rules(both, buckets, distance):
    tk = 300 if distance < 2048 else 2500
    shape = (1, 2, 6, tk)
    scores = torch.zeros(shape, device="cuda")
    table = torch.randn(buckets, 2, generator=torch.Generator().manual_seed(1)).cuda()
    start = [tk // 2]
    check_forward(scores, table, distance, both, q_start=start)
    check_backward(scores, table, distance, both, q_start=start, dprobs=make(*shape, torch.float32, seed=2, sigma=1.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_masks_and_empty_rows(dtype):
    b, h, tq, tk = 4, 2, 37, 130
    scores = make(b, h, tq, tk, dtype, seed=8)
    dprobs = make(b, h, tq, tk, dtype, seed=9, sigma=1.0)
    table = torch.randn(32, h, generator=torch.Generator().manual_seed(3)).cuda()
    k_len = [0, 1, 64, 500]
    start = [0, -5, 20, 90]     # -5: the first five queries see no key when causal
    # what is not seen may hold anything
    for ib in range(b):
        scores[ib, :, :, min(k_len[ib], tk):] = math.nan
        dprobs[ib, :, :, min(k_len[ib], tk):] = math.inf
    clean_s, clean_d = torch.nan_to_num(scores, 0, 0, 0), torch.nan_to_num(dprobs, 0, 0, 0)
    dev = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    for causal in (False, True):
        p, stats = check_forward(clean_s, table, 100, False, causal, 0.5, k_len, start)
        p2, stats2 = bz.bias_softmax(scores, table, 100, False, causal, 0.5, dev(k_len), dev(start))
        assert torch.equal(p, p2) and torch.equal(stats, stats2)
        assert (p[0] == 0).all() and (stats[0, ..., 0] == -math.inf).all()
        ds, dt = check_backward(clean_s, table, 100, False, causal, 0.5, k_len, start, clean_d)
        ds2, dt2 = bz.bias_softmax_backward(scores, table, stats, dprobs, 100, False, causal, 0.5, dev(k_len), dev(start))
        assert torch.equal(ds, ds2) and torch.equal(dt, dt2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_values_at_the_ends(dtype):
    tk = 70
    scores = torch.zeros(1, 1, 6, tk, dtype=dtype)
    lowest = torch.finfo(dtype).min
    scores[0, 0, 0, 3:] = -math.inf          # three keys left
    scores[0, 0, 1, :] = -math.inf           # none
    scores[0, 0, 2, 5:] = lowest             # masked with the type's lowest value
    scores[0, 0, 3, :] = lowest              # all of them: still a distribution
    scores[0, 0, 4, :] = -1000.0             # far below zero, all alike but a few at -inf
    scores[0, 0, 4, 1::2] = -math.inf
    scores[0, 0, 5, 7] = math.nan
    scores = scores.cuda()
    table = torch.zeros(8, 1, device="cuda")
    p, stats = bz.bias_softmax(scores, table, 16, True)
    p = p.float().cpu()[0, 0]
    lse = log_sum(stats)[0, 0]
    unit = HALF_UNIT[dtype] + P_TOL
    assert torch.allclose(p[0, :3], torch.full((3,), 1 / 3), rtol=unit) and (p[0, 3:] == 0).all()
    assert (p[1] == 0).all() and lse[1] == -math.inf
    assert torch.allclose(p[2, :5], torch.full((5,), 0.2), rtol=unit) and (p[2, 5:] == 0).all()
    assert torch.allclose(p[3], torch.full((tk,), 1 / tk), rtol=unit)
    assert torch.allclose(p[4, ::2], torch.full((tk // 2,), 2 / tk), rtol=unit) and (p[4, 1::2] == 0).all()
    assert torch.isnan(p[5]).all() and torch.isnan(lse[5])
    dprobs = torch.ones_like(scores)
    ds, _ = bz.bias_softmax_backward(scores, table, stats, dprobs, 16, True)
    ds = ds.float().cpu()[0, 0]
    assert (ds[1] == 0).all() and torch.isfinite(ds[:5]).all() and ds[:5].abs().max() < 1e-3


@pytest.mark.parametrize("tk", [777, 784])
def test_single_query_behind_a_cache(tk):
    b, h = 5, 4
    k_len = [1, 2, 128, 500, tk]
    for dtype in (torch.float16, torch.float32):
        scores = make(b, h, 1, tk, dtype, seed=4)
        table = torch.randn(32, h, generator=torch.Generator().manual_seed(3)).cuda()
        last, _ = check_forward(scores, table, 128, False, False, 1.0, k_len, [n - 1 for n in k_len])
        # the same row out of a causal block that ends there
        wide = scores.expand(b, h, 3, tk).contiguous()
        block, _ = check_forward(wide, table, 128, False, True, 1.0, k_len, [n - 3 for n in k_len])
        if tk % 16 == 0:    # rows that sit alike: the same order of sums
            assert torch.equal(block[:, :, 2:], last)


def test_in_place_other_stream_and_same_bits():
    scores, dprobs = make(2, 4, 100, 515, torch.bfloat16, seed=1), make(2, 4, 100, 515, torch.bfloat16, seed=2)
    table = torch.randn(32, 4, generator=torch.Generator().manual_seed(3)).cuda()
    p, stats = bz.bias_softmax(scores, table)
    ds, dt = bz.bias_softmax_backward(scores, table, stats, dprobs)
    for _ in range(20):
        p2, _ = bz.bias_softmax(scores, table)
        ds2, dt2 = bz.bias_softmax_backward(scores, table, stats, dprobs)
        assert torch.equal(p, p2) and torch.equal(ds, ds2) and torch.equal(dt, dt2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a, d = scores.clone(), dprobs.clone()
        bz.bias_softmax_backward(a, table, stats, d, dscores=d)
        bz.bias_softmax(a, table, probs=a)
    s.synchronize()
    assert torch.equal(a, p) and torch.equal(d, ds)


def test_gradient_against_differences():
    """Central differences of sum(p * c) in 64 bits at the table and at scores (the formula itself), and the kernel's
    gradient against them: step 1e-4 gives the difference an error of about 1e-7."""
    b, h, tq, tk = 1, 2, 4, 9
    scores, c = make(b, h, tq, tk, torch.float32, seed=1, sigma=1.0), make(b, h, tq, tk, torch.float32, seed=2, sigma=1.0)
    table = torch.randn(8, h, generator=torch.Generator().manual_seed(3)).cuda()
    _, stats = bz.bias_softmax(scores, table, 6, True, scale=0.7)
    ds, dt = bz.bias_softmax_backward(scores, table, stats, c, 6, True, scale=0.7)
    value = lambda s, t: float((reference(s, t, 6, True, False, 0.7, None, None)[0] * c.cpu().double()).sum())  # noqa: E731
    step = 1e-4
    for where in [(0, 0, 0, 0), (0, 1, 2, 5), (0, 0, 3, 8)]:
        up, down = scores.cpu().double(), scores.cpu().double()
        up[where] += step
        down[where] -= step
        assert abs((value(up, table) - value(down, table)) / (2 * step) - float(ds[where])) < 5e-6
    for where in [(0, 0), (3, 1), (4, 0), (5, 1), (7, 0)]:
        up, down = table.cpu().double(), table.cpu().double()
        up[where] += step
        down[where] -= step
        assert abs((value(scores, up) - value(scores, down)) / (2 * step) - float(dt[where])) < 5e-6


def test_only_what_is_asked_for():
    scores, dprobs = make(1, 2, 8, 40, torch.float32, seed=1), make(1, 2, 8, 40, torch.float32, seed=2)
    table = torch.randn(8, 2, generator=torch.Generator().manual_seed(3)).cuda()
    _, stats = bz.bias_softmax(scores, table, 20, True)
    ds, dt = bz.bias_softmax_backward(scores, table, stats, dprobs, 20, True)
    st = (bz._strides(scores, "s"))
    ds2, dt2 = torch.zeros_like(ds), torch.zeros_like(dt)
    ws = torch.empty(bz.lib().bz_bias_softmax_workspace_bytes(1, 2, 8, 40, 8), dtype=torch.uint8, device="cuda")
    common = (scores.data_ptr(), st, bz.F32, 1, 2, 8, 40, table.data_ptr(), 8, 20, 1, 0, 1.0, None, None, stats.data_ptr(), dprobs.data_ptr(), st)
    assert bz.lib().bz_bias_softmax_backward(*common, ds2.data_ptr(), st, None, None, 0, None) == bz.OK
    assert bz.lib().bz_bias_softmax_backward(*common, None, None, dt2.data_ptr(), ws.data_ptr(), ws.numel(), None) == bz.OK
    torch.cuda.synchronize()
    assert torch.equal(ds, ds2) and torch.equal(dt, dt2)


@pytest.mark.parametrize("both,buckets,distance,at", [(False, 73, 905, 347), (False, 109, 1549, 183), (True, 218, 1549, 183), (False, 187, 1839, 96), (False, 226, 188, 157)])
def test_distances_next_to_a_bound_just_above_them(both, buckets, distance, at):
    """The bound of a bucket lies a billionth above the distance `at`, which still belongs to the bucket before."""
    shape = (1, 2, 3, 9)
    scores = make(*shape, torch.float32, seed=at)
    table = torch.randn(buckets, 2, generator=torch.Generator().manual_seed(at)).cuda()
    check_forward(scores, table, distance, both, q_start=[at + 1])
    check_backward(scores, table, distance, both, q_start=[at + 1], dprobs=make(*shape, torch.float32, seed=1 + at, sigma=1.0))


def test_no_keys_at_all():
    table = torch.randn(32, 2, device="cuda")
    for given in (None, torch.full((1, 2, 3, 2), 5.0, device="cuda")):
        probs, stats = bz.bias_softmax(torch.empty(1, 2, 3, 0, device="cuda"), table, stats=given)
        assert probs.shape == (1, 2, 3, 0) and (stats[..., 0] == -math.inf).all() and (stats[..., 1] == 0).all()
    ds, dt = bz.bias_softmax_backward(torch.empty(1, 2, 3, 0, device="cuda"), table, stats, torch.empty(1, 2, 3, 0, device="cuda"))
    assert ds.shape == (1, 2, 3, 0) and (dt == 0).all()
