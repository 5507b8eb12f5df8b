"""bz_glu and bz_glu_backward against the formulas in 64 bits.

Tolerances, element by element.  A sum of L products of 16-bit values is held in 32 bits; the products are exact, and
each of the L/8 + 16 additions into the running sum (the tensor core adds at least 8 products at a time and may drop bits
below the last place) costs at most 2^-23 of the sum of the terms' sizes: eps(L) = (L/8 + 16) * 2^-23.  The
activation's exponential costs 1e-5 relative at most for |g| < 20.  dg and du are rounded to the inputs' type before the
products (half a unit; 2^-25 absolute in binary16's subnormal range), results once more when they are stored.
"""
import math

import pytest
import torch

from paper_2010_04902_b200 import binding as bz

pytestmark = pytest.mark.gpu

HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
FLOOR = {torch.float32: 1e-37, torch.float16: 2.0 ** -25, torch.bfloat16: 1e-37}
ACTS = ["silu", "gelu_tanh", "gelu", "relu"]


def eps(L):
    return (L / 8 + 16) * 2.0 ** -23


def act(name, g):
    """Activation and slope in 64 bits."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "relu":
        return g.clamp(min=0), (g > 0).double()
    if name == "gelu":
        phi = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
        return g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def make(m, n, k, dtype, seed, pad_x=0, pad_w=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    wide = lambda r, c, pad, s: (torch.randn(r, c + pad, generator=gen) * s).to(dtype).cuda()[:, :c]  # noqa: E731
    x = wide(m, k, pad_x, scale)
    wg, wu = wide(n, k, pad_w, max(k, 1) ** -0.5), wide(n, k, pad_w, max(k, 1) ** -0.5)
    return x, wg, wu, wide(m, n, 0, 1.0)


def check(x, wg, wu, dh, name, **kw):
    m, k = x.shape
    n = wg.shape[0]
    dt = x.dtype
    hu, fl = HALF_UNIT[dt], FLOOR[dt]
    preact = torch.full((2, m, n), math.nan, dtype=torch.float32, device="cuda")
    h = bz.glu(x, wg, wu, name, preact=preact)
    assert torch.equal(h, bz.glu(x, wg, wu, name))
    X, G, U, D = (t.double() for t in (x, wg, wu, dh))
    g, u = X @ G.T, X @ U.T
    dg_, du_ = eps(k) * (X.abs() @ G.abs().T), eps(k) * (X.abs() @ U.abs().T)
    assert ((preact[0].double() - g).abs() <= dg_ + 1e-30).all() and ((preact[1].double() - u).abs() <= du_ + 1e-30).all()
    a, s = act(name, g)
    # |act'| <= 1.13, |act''| <= 1.6 for the smooth ones; where relu's g is within its error of 0 both slopes are right
    ea = 1.2 * dg_ + 1e-5 * a.abs() + 1e-7
    eh = ea * (u.abs() + du_) + (a.abs() + ea) * du_
    want = a * u
    assert ((h.double() - want).abs() <= eh + hu * (want.abs() + eh) + fl).all()
    # the gradient is checked from the projections that the forward call kept
    dx, dwg, dwu = bz.glu_backward(x, wg, wu, preact, dh, name, **kw)
    a, s = act(name, preact[0].double())
    es = 2e-5
    P, Q = D * preact[1].double() * s, D * a
    eP = hu * P.abs() + es * (D * preact[1].double()).abs() + fl
    eQ = hu * Q.abs() + es * (D.abs() * (a.abs() + 0.01)) + fl
    want = P @ G + Q @ U
    size = P.abs() @ G.abs() + Q.abs() @ U.abs()
    bound = eP @ G.abs() + eQ @ U.abs() + eps(2 * n) * size
    assert ((dx.double() - want).abs() <= 1.01 * bound + hu * want.abs() + fl).all()
    hw, fw = HALF_UNIT[dwg.dtype], FLOOR[dwg.dtype]
    for got, A, E in ((dwg, P, eP), (dwu, Q, eQ)):
        want = A.T @ X
        bound = E.T @ X.abs() + eps(m) * (A.abs().T @ X.abs())
        assert ((got.double() - want).abs() <= 1.01 * bound + hw * want.abs() + fw).all()
    return h, dx, dwg, dwu


SHAPES = [(1, 1, 1), (1, 8, 8), (2, 3, 5), (1, 130, 64), (3, 257, 200), (16, 64, 512), (17, 100, 96), (33, 129, 72), (64, 128, 64), (65, 136, 136),
          (100, 300, 1000), (128, 128, 128), (129, 257, 65), (256, 256, 256), (300, 1000, 520), (777, 130, 264), (1000, 64, 1032)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_matches(shape, dtype):
    m, n, k = shape
    check(*make(m, n, k, dtype, seed=m + n + k), ACTS[(m + n + k) % 4])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", [(2048, 4100, 136), (2050, 4104, 1032), (4096, 2048, 1024), (9000, 600, 520)])
def test_more_tiles_than_clusters(shape, dtype):
    """The widest tiles and several rounds of them, whole and ragged."""
    m, n, k = shape
    check(*make(m, n, k, dtype, seed=m + n + k), ACTS[(m + n) % 4])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(1, 2048, 1024), (1, 5461, 2048), (8, 5461, 776), (9, 1030, 2049 // 8 * 8), (17, 2500, 1001), (24, 4001, 513), (25, 3001, 2000), (32, 2400, 4104)])
def test_few_rows_and_many_weights(m, n, k, dtype):
    """The ring; 1001 and 513 lie off the 16-byte grid (or are made to fit by a stride)."""
    check(*make(m, n, k, dtype, seed=m + n + k), ACTS[(m + n) % 4])
    check(*make(m, n, k, dtype, seed=m + n + k, pad_w=-k % 8, pad_x=-k % 8), ACTS[n % 4])


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("m", [2, 200])
def test_activations(name, m):
    check(*make(m, 200, 64, torch.bfloat16, seed=1, scale=3.0), name)


@pytest.mark.parametrize("m", [1, 40, 150])
@pytest.mark.parametrize("pad_x,pad_w", [(8, 0), (0, 16), (1, 0), (0, 3), (5, 7)])
def test_strides(m, pad_x, pad_w):
    x, wg, wu, dh = make(m, 90, 104, torch.float16, seed=pad_x + 10 * pad_w, pad_x=pad_x, pad_w=pad_w)
    check(x, wg, wu, dh, "silu")


@pytest.mark.parametrize("m", [1, 40, 150])
def test_bases_off_their_boundary(m):
    x, wg, wu, dh = make(m, 96, 104, torch.bfloat16, seed=4)
    off = lambda t: torch.cat([torch.zeros(3, dtype=t.dtype, device="cuda"), t.reshape(-1)])[3:].view(t.shape)  # noqa: E731
    a = check(x, wg, wu, dh, "silu")
    b = check(off(x), off(wg), off(wu), off(dh), "silu")
    for p, q in zip(a, b):
        assert torch.equal(p, q)    # laid out on the way in, then the same kernels


@pytest.mark.parametrize("n,k", [(90, 104), (91, 103), (64, 128)])
def test_outputs_into_wider_buffers(n, k):
    m = 70
    x, wg, wu, dh = make(m, n, k, torch.float16, seed=6)
    h0 = bz.glu(x, wg, wu, "gelu")
    for pad, at in ((0, 0), (6, 3), (16, 8)):
        buf = torch.full((m, n + pad), 7.0, dtype=torch.float16, device="cuda")
        bz.glu(x, wg, wu, "gelu", h=buf[:, at:at + n])
        assert torch.equal(buf[:, at:at + n], h0) and (buf[:, :at] == 7).all() and (buf[:, at + n:] == 7).all()
    preact = torch.empty(2, m, n, device="cuda")
    bz.glu(x, wg, wu, "gelu", preact=preact)
    dx0, dg0, du0 = bz.glu_backward(x, wg, wu, preact, dh, "gelu")
    for pad, at in ((6, 3), (16, 8)):
        big = lambda r, c, dt: torch.full((r, c + pad), 7.0, dtype=dt, device="cuda")  # noqa: E731
        bx, bg, bu = big(m, k, torch.float16), big(n, k, torch.float16), big(n, k, torch.float16)
        cut = lambda t, c: t[:, at:at + c]  # noqa: E731
        bz.glu_backward(x, wg, wu, preact, dh, "gelu", dx=cut(bx, k), dw_gate=cut(bg, k), dw_up=cut(bu, k))
        for buf, want in ((bx, dx0), (bg, dg0), (bu, du0)):
            assert torch.equal(cut(buf, k), want) and (buf[:, :at] == 7).all() and (buf[:, at + k:] == 7).all()


@pytest.mark.parametrize("m,n,k", [(64, 40, 24), (50, 33, 17), (700, 260, 264)])
def test_weight_gradients_in_a_gradient_row(m, n, k):
    """binary32 gradients written into a file's row at an odd place: the 32-bit sums, unrounded."""
    x, wg, wu, dh = make(m, n, k, torch.bfloat16, seed=m)
    row = torch.full((2 * n * k + 11,), 7.0, device="cuda")
    dwg, dwu = row[5:5 + n * k].view(n, k), row[5 + n * k:5 + 2 * n * k].view(n, k)
    _, _, a, b = check(x, wg, wu, dh, "silu", dw_gate=dwg, dw_up=dwu)
    assert (row[:5] == 7).all() and (row[5 + 2 * n * k:] == 7).all()
    preact = torch.empty(2, m, n, device="cuda")
    bz.glu(x, wg, wu, "silu", preact=preact)
    _, c, d = bz.glu_backward(x, wg, wu, preact, dh, "silu")
    assert torch.equal(a.to(torch.bfloat16), c) and torch.equal(b.to(torch.bfloat16), d)


def test_nothing_and_empty_sums():
    x, wg, wu, dh = make(5, 7, 0, torch.float16, seed=1)
    preact = torch.full((2, 5, 7), 3.0, device="cuda")
    assert (bz.glu(x, wg, wu, preact=preact) == 0).all() and (preact == 0).all()
    dx, dg, du = bz.glu_backward(x, wg, wu, preact, dh)
    assert dx.numel() == dg.numel() == du.numel() == 0
    x, wg, wu, dh = make(0, 7, 9, torch.float16, seed=1)
    assert bz.glu(x, wg, wu).numel() == 0
    dg, du = torch.ones(7, 9, dtype=torch.float16, device="cuda"), torch.ones(7, 9, dtype=torch.float16, device="cuda")
    bz.glu_backward(x, wg, wu, torch.empty(2, 0, 7, device="cuda"), dh, dw_gate=dg, dw_up=du)
    assert (dg == 0).all() and (du == 0).all()
    x, wg, wu, dh = make(5, 0, 9, torch.float16, seed=1)
    dx = torch.ones(5, 9, dtype=torch.float16, device="cuda")
    bz.glu_backward(x, wg, wu, torch.empty(2, 5, 0, device="cuda"), dh, dx=dx)
    assert (dx == 0).all()


def test_infinities_and_nan_stay_in_their_rows():
    x, wg, wu, dh = make(200, 96, 64, torch.bfloat16, seed=2)
    clean = bz.glu(x, wg, wu)
    x[7, 3], x[150, 0] = math.nan, math.inf
    got = bz.glu(x, wg, wu)
    assert torch.isnan(got[7]).all() and not torch.isfinite(got[150]).all()
    keep = [i for i in range(200) if i not in (7, 150)]
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("m,n,k", [(4, 300, 512), (32, 2400, 4104), (300, 264, 264), (2000, 136, 72)])
def test_same_bits_every_time_and_on_another_stream(m, n, k):
    x, wg, wu, dh = make(m, n, k, torch.bfloat16, seed=3)
    preact = torch.empty(2, m, n, device="cuda")
    first = (bz.glu(x, wg, wu, preact=preact),) + bz.glu_backward(x, wg, wu, preact, dh)
    for _ in range(100):   # a stage refilled too early showed in one run of twenty (32 rows, contraction 4104)
        again = (bz.glu(x, wg, wu, preact=preact),) + bz.glu_backward(x, wg, wu, preact, dh)
        assert all(torch.equal(p, q) for p, q in zip(first, again))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = (bz.glu(x, wg, wu, preact=preact),) + bz.glu_backward(x, wg, wu, preact, dh)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, again))


def test_gradient_against_differences():
    """Central differences of sum(h * dh) in 64 bits, with steps that the inputs' type holds exactly (2^-6: the
    difference is off by the third derivative's share, about 1e-4 of the gradient's scale), and the kernel's gradient:
    binary16 operands, so half a unit (2^-11) of the terms' sizes (about 10 here) on top."""
    x, wg, wu, dh = make(3, 8, 8, torch.float16, seed=9)
    preact = torch.empty(2, 3, 8, device="cuda")
    bz.glu(x, wg, wu, "gelu_tanh", preact=preact)
    grads = bz.glu_backward(x, wg, wu, preact, dh, "gelu_tanh")
    step = 2.0 ** -6

    def value(t):
        X, G, U = t
        return float((act("gelu_tanh", X @ G.T)[0] * (X @ U.T) * dh.double()).sum())

    for which, grad in enumerate(grads):
        for where in [(0, 0), (2, 5), (1, 7)]:
            up, down = [t.double().clone() for t in (x, wg, wu)], [t.double().clone() for t in (x, wg, wu)]
            up[which][where] += step
            down[which][where] -= step
            assert abs((value(up) - value(down)) / (2 * step) - float(grad[where])) < 0.02


def test_only_what_is_asked_for():
    x, wg, wu, dh = make(40, 48, 56, torch.float16, seed=9)
    preact = torch.empty(2, 40, 48, device="cuda")
    bz.glu(x, wg, wu, preact=preact)
    dx, dg, du = bz.glu_backward(x, wg, wu, preact, dh)
    ws = torch.empty(bz.glu_workspace_bytes(40, 48, 56, torch.float16, True), dtype=torch.uint8, device="cuda")
    dx2, dg2, du2 = torch.zeros_like(dx), torch.zeros_like(dg), torch.zeros_like(du)
    head = (x.data_ptr(), 56, wg.data_ptr(), wu.data_ptr(), 56, preact.data_ptr(), dh.data_ptr(), 48, 40, 48, 56, bz.F16, bz.ACT_SILU)
    tail = (bz.F16, ws.data_ptr(), ws.numel(), None)
    assert bz.lib().bz_glu_backward(*head, dx2.data_ptr(), 56, None, None, 0, *tail) == bz.OK
    assert bz.lib().bz_glu_backward(*head, None, 0, dg2.data_ptr(), du2.data_ptr(), 56, *tail) == bz.OK
    torch.cuda.synchronize()
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2) and torch.equal(du, du2)


def test_stages_of_the_ring_are_not_refilled_under_their_readers():
    """Weights that are one number for each group of eight units (gate +, up -, exact in every sum) and tokens that mark parts
    of the contraction: a product that took a later group's weights shows in whichever call it happens (one in a million
    before the readers fenced, at these sizes)."""
    n, k = 5461, 2048
    group = torch.arange(n, device="cuda") // 8
    code = (128 + group % 128).float() * 2.0 ** (group // 128).float()
    wg = code[:, None].expand(n, k).to(torch.bfloat16).contiguous()
    wu = -wg
    at = torch.arange(k, device="cuda")
    x = torch.stack([at // 256 == i for i in range(8)] + [at % 256 // 32 == i for i in range(8)] + [at % 8 == i for i in range(8)]).to(torch.bfloat16)
    want = torch.stack([x.float().sum(1)[:, None] * code, -x.float().sum(1)[:, None] * code])
    preact, h = torch.empty(2, 24, n, device="cuda"), torch.empty(24, n, dtype=torch.bfloat16, device="cuda")
    differs = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(20000):
        bz.glu(x, wg, wu, h=h, preact=preact)
        differs += (preact != want).any()
    assert int(differs) == 0


@pytest.mark.parametrize("m", [8, 89])
def test_gelu_far_below_zero(m):
    """act(g) and its slope for g in [-10, 4.75], exact in bfloat16, relative to their own size: the erfc's argument is known
    to 2^-23 relative, which its exponential makes g^2 2^-23 (1.2e-5 at -10), and the fast exponential of the slope adds
    50 units of 2^-23 at most; then half a unit of the type.  Near its zero (g about -0.75) the slope is a difference
    of terms of 0.2.  h = act * 1; dx's two columns are dg = dh * 1 * slope and du = dh * act."""
    g = (torch.arange(m, device="cuda", dtype=torch.float64) / 6 - 10).to(torch.bfloat16)
    x = torch.stack([g, torch.ones_like(g)], 1).contiguous()
    wg, wu = torch.tensor([[1.0, 0.0]], device="cuda").to(torch.bfloat16), torch.tensor([[0.0, 1.0]], device="cuda").to(torch.bfloat16)
    preact, dh = torch.empty(2, m, 1, device="cuda"), torch.ones(m, 1, dtype=torch.bfloat16, device="cuda")
    h = bz.glu(x, wg, wu, "gelu", preact=preact)
    dx, _, _ = bz.glu_backward(x, wg, wu, preact, dh, "gelu")
    G = g.double()
    phi, density = 0.5 * torch.special.erfc(-G / math.sqrt(2)), torch.exp(-G * G / 2) / math.sqrt(2 * math.pi)
    want, slope = G * phi, phi + G * density
    near = 2.0 ** -8 + 2e-5
    assert ((h[:, 0].double() - want).abs() <= near * want.abs()).all()
    assert ((dx[:, 1].double() - want).abs() <= near * want.abs()).all()
    assert ((dx[:, 0].double() - slope).abs() <= 2.0 ** -8 * slope.abs() + 2e-5 * (phi + (G * density).abs())).all()


def test_longest_contraction():
    """One tile whose contraction alone takes longer than a second (2^28 elements, 19 GB): nothing may run out meanwhile."""
    m, n, k = 33, 1, 1 << 28
    x = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
    wg, wu = torch.zeros(n, k, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, k, dtype=torch.bfloat16, device="cuda")
    for at, (a, b) in {0: (1.0, 3.0), 12345677: (2.0, 5.0), k - 1: (4.0, 7.0)}.items():
        x[:, at] = torch.arange(m, device="cuda") + 1
        wg[:, at], wu[:, at] = a, b
    preact = torch.empty(2, m, n, device="cuda")
    h = bz.glu(x, wg, wu, "relu", preact=preact)
    row = (torch.arange(m, device="cuda") + 1).float()[:, None]
    assert torch.equal(preact, torch.stack([7 * row, 15 * row])) and torch.equal(h, (105 * row * row).to(torch.bfloat16))
