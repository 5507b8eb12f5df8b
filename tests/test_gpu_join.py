"""bz_join and bz_join_backward against the formulas in 64 bits.

Tolerances.  Forward: s is three binary32 products and a sum, the norms' 1 / deviation a sum of n squares (relative error below
2^-24 (log2 n + n / 32 / 2) by their tree; 2e-6 covers 16384 columns), so values are known to 4e-6 of the sum of their terms' sizes, and half a
unit of the type.  For a layer norm the size is that of the value plus its row's mean.  Backward: the same per term, where the normalised stream carries the error of s (4e-6 of the sizes of its terms) too.
Column sums over m rows in binary32: 2^-24 * (rows of a CTA + CTAs) of the sum of sizes, below 2e-5 here.
"""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from test_gpu_dropout import kept

pytestmark = pytest.mark.gpu

HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}
TOL, SUM_TOL = 4e-6, 2e-5
EPS = 1e-6
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def wide(m, n, pad, dtype, g, sigma=1.0, mean=0.0):
    full = torch.empty(m, n + pad, dtype=dtype, device="cuda")
    full[:, :n] = (torch.randn(m, n, generator=g) * sigma + mean).to(dtype).cuda()
    return full[:, :n]


def make(m, n, dtype, seed=0, pad=0, post=True, pre=True, groups=1, rate=0.1, norm="rms", branch=True, residual=1.0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    w = lambda *shape: (torch.randn(*shape, generator=g) * 0.2 + 1).cuda()  # noqa: E731
    t = {"x": wide(m, n, pad, dtype, g, 2.0, 0.3), "y": wide(m, n, pad, dtype, g, 0.7, -0.2) if branch else None,
         "ds": wide(m, n, pad, dtype, g), "dz": wide(m, n, pad, dtype, g) if pre else None}
    form = {"w_post": w(n) if post else None, "gate": w(groups, n) if groups else None, "w_pre": w(n) if pre else None, "norm": norm,
            "residual_scale": residual, "branch_scale": scale, "rate": rate, "rng": torch.tensor([seed + 11, 3], device="cuda") if rate else None}
    return t, form


def normed(v, kind):
    """(normalised rows, 1 / deviation, size of the values before the mean went)."""
    size = v.abs()
    if kind == "layer":
        mean = v.mean(1, keepdim=True)
        size = size + mean.abs()
        v = v - mean
    r = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r, size * r


def normed_backward(d, hat, r, kind):
    """(gradient, size of its terms)."""
    c1, s1 = (d * hat).mean(1, keepdim=True), (d * hat).abs().mean(1, keepdim=True)
    out, size = d - hat * c1, d.abs() + hat.abs() * s1
    if kind == "layer":
        out, size = out - d.mean(1, keepdim=True), size + d.abs().mean(1, keepdim=True)
    return out * r, size * r


def reference(t, form):
    """Every output with the sum of its terms' sizes."""
    host = lambda v: None if v is None else v.detach().cpu().double()  # noqa: E731
    x, y, ds, dz = (host(t[k]) for k in ("x", "y", "ds", "dz"))
    w_post, gate, w_pre = (host(form[k]) for k in ("w_post", "gate", "w_pre"))
    m, n = x.shape
    kind, groups = form["norm"], 0 if gate is None else gate.shape[0]
    s, size = form["residual_scale"] * x, (form["residual_scale"] * x).abs()
    out = {}
    if y is not None:
        hat, _, hat_size = normed(y, kind) if w_post is not None else (y, None, y.abs())
        a = hat * w_post if w_post is not None else hat
        a_size = hat_size * w_post.abs() if w_post is not None else hat_size
        f = torch.full((m, n), form["branch_scale"], dtype=torch.float64)
        if form["rate"]:
            t16 = round(form["rate"] * 65536)
            f = f * kept(form["rng"].tolist(), m * n, form["rate"]).view(m, n) * (65536 / (65536 - t16))
        gated = f * gate.repeat_interleave(m // groups, 0) if groups else f
        s, size = s + gated * a, size + (gated * a_size).abs()
    out["s"] = (s, size)
    if w_pre is not None:
        pre_hat, r_s, pre_size = normed(s, kind)
        out["z"] = (pre_hat * w_pre, (size + (s.mean(1, keepdim=True).abs() if kind == "layer" else 0)) * r_s * w_pre.abs() + pre_size * w_pre.abs())
    g = ds if ds is not None else torch.zeros_like(x)
    g_size = g.abs()
    if w_pre is not None:
        out["dw_pre"] = (torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64))
    if dz is not None:
        hat, r, hat_size = normed(s, kind)
        hat_size = hat_size + size * r        # what s was summed from
        dpre, _ = normed_backward(dz * w_pre, hat, r, kind)
        dsize = normed_backward(dz * w_pre, hat_size, r, kind)[1]
        g, g_size = g + dpre, g_size + dsize
        out["dw_pre"] = ((dz * hat).sum(0), (dz.abs() * hat_size).sum(0))
    rs = abs(form["residual_scale"])
    out["dx"] = (form["residual_scale"] * g, rs * g_size)
    if y is not None:
        u, u_size = f * g, f.abs() * g_size
        if groups:
            per = lambda v: v.view(groups, m // groups, n).sum(1)  # noqa: E731
            out["dgate"] = (per(u * a), per(u_size * a_size))
            wide_gate = gate.repeat_interleave(m // groups, 0)
            u, u_size = u * wide_gate, u_size * wide_gate.abs()
        if w_post is not None:
            hat, r, hat_size = normed(y, kind)
            out["dw_post"] = ((u * hat).sum(0), (u_size * hat_size).sum(0))
            dy, _ = normed_backward(u * w_post, hat, r, kind)
            e = u_size * w_post.abs()
            out["dy"] = (dy, r * (e + hat_size * (e * hat_size).mean(1, keepdim=True) + (e.mean(1, keepdim=True) if kind == "layer" else 0)))
        else:
            out["dy"] = (u, u_size)
    return out


def near(got, want, tol, half=0.0, tiny=0.0):
    value, size = want
    return bool(((got.cpu().double() - value).abs() <= tol * size + half * value.abs() + tiny).all())


def check(t, form, into=None):
    dtype = t["x"].dtype
    half, tiny = HALF_UNIT[dtype], TINY[dtype]
    into = into or {}
    s, z, stats = bz.join(t["x"], t["y"], **form, eps=EPS, **{k: into[k] for k in ("s", "z") if k in into})
    want = reference(t, form)
    assert near(s, want["s"], TOL, half, tiny)
    assert (z is None) == (form["w_pre"] is None)
    if z is not None:
        assert near(z, want["z"], TOL, half, tiny)
    got = dict(zip(("dx", "dy", "dw_post", "dgate", "dw_pre"),
                   bz.join_backward(t["x"], t["y"], stats, ds=t["ds"], dz=t["dz"], **form, **{k: into[k] for k in ("dx", "dy") if k in into})))
    for name, value in got.items():
        assert (value is None) == (name not in want), name
        if value is None:
            continue
        if name in ("dx", "dy"):
            assert near(value, want[name], TOL, half, tiny), name
        else:
            assert value.dtype == torch.float32 and near(value, want[name], SUM_TOL, 0.0, 1e-30), name
    return s, z, stats, got


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 64), (3, 2), (5, 33), (2, 264), (9, 1000), (4, 1001), (3, 4096), (2, 5000), (2, 8192), (2, 8200), (1, 16384), (3, 16383)])
def test_matches(m, n, norm, dtype):
    check(*make(m, n, dtype, seed=n, norm=norm, residual=1.3, scale=0.8))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,groups,pad", [(777, 264, 3, 0), (1200, 120, 1, 8), (2048, 64, 64, 0), (333, 1001, 333, 0), (700, 515, 7, 5), (450, 2056, 1, 0), (400, 4096, 2, 0),
                                            (310, 8192, 1, 0), (301, 9000, 7, 0), (2500, 40, 2500, 3)])
def test_many_rows(m, n, groups, pad, dtype):
    t, form = make(m, n, dtype, seed=m, pad=pad, groups=groups, norm="layer" if m % 2 else "rms")
    s, z, stats, got = check(t, form)
    for _ in range(10):
        again = bz.join(t["x"], t["y"], **form, eps=EPS)
        back = bz.join_backward(t["x"], t["y"], stats, ds=t["ds"], dz=t["dz"], **form)
        assert torch.equal(again[0], s) and torch.equal(again[1], z) and torch.equal(again[2], stats)
        assert all(torch.equal(a, b) for a, b in zip(back, got.values()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [96, 777, 2048, 10000])
@pytest.mark.parametrize("change", [dict(post=False), dict(pre=False), dict(groups=0), dict(rate=0.0), dict(post=False, groups=0, rate=0.0), dict(post=False, pre=False, groups=0),
                                    dict(branch=False, post=False, groups=0, rate=0.0), dict(branch=False, post=False, groups=0, rate=0.0, residual=0.5, norm="layer"),
                                    dict(rate=0.75, scale=-2.0, groups=6), dict(residual=0.0)])
def test_forms(change, n, dtype):
    check(*make(6, n, dtype, seed=1, **change))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,pad", [(1900, 600, 0), (1900, 768, 0), (1300, 1536, 0), (600, 2304, 8), (600, 2560, 0), (600, 2561, 0), (400, 4600, 8), (400, 5120, 0), (400, 5128, 0),
                                     (310, 6144, 8), (310, 6143, 2), (310, 6152, 0), (300, 7000, 0), (160, 9600, 0), (160, 12288, 0), (160, 13000, 0), (150, 12281, 0)])
def test_widths_between_powers_of_two(m, n, pad, dtype):
    """A CTA's threads are what such a row needs, or more; several of them share an SM and take some rows one after the other."""
    check(*make(m, n, dtype, seed=n, pad=pad, norm="layer" if m % 100 else "rms"))


@pytest.mark.parametrize("which", ["ds", "dz"])
def test_one_gradient_alone(which):
    t, form = make(10, 300, torch.bfloat16, seed=2)
    t[which] = None
    check(t, form)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("n,pad,where", [(1000, 1, 0), (515, 5, 3), (2048, 8, 8), (8192, 4, 4)])
def test_rows_that_sit_differently(n, pad, where, dtype):
    t, form = make(150, n, dtype, seed=3, pad=pad)
    outer = {k: torch.full((150, n + 70), 7.0, dtype=dtype, device="cuda") for k in ("s", "z", "dx", "dy")}
    check(t, form, {k: v[:, where:where + n] for k, v in outer.items()})
    for v in outer.values():
        assert (v[:, :where] == 7).all() and (v[:, where + n:] == 7).all()


def test_the_norm_alone_leaves_its_input():
    t, form = make(20, 512, torch.bfloat16, seed=4, branch=False, post=False, groups=0, rate=0.0)
    s, z, stats = bz.join(t["x"], w_pre=form["w_pre"])
    assert s is t["x"] and z.shape == s.shape
    dx, dy, dw_post, dgate, dw_pre = bz.join_backward(t["x"], None, stats, dz=t["dz"], w_pre=form["w_pre"])
    assert dy is None and dw_post is None and dgate is None and dw_pre.shape == (512,)


def test_dropout_is_that_of_the_call_for_it():
    m, n = 31, 517
    x, y = torch.zeros(m, n, device="cuda"), torch.randn(m, n, device="cuda")
    rng = torch.tensor([5, 6], device="cuda")
    s, _, _ = bz.join(x, y, rate=0.3, rng=rng)
    assert torch.equal(s, bz.dropout(y, 0.3, rng))


def test_zero_rows_and_large_values():
    """A row of zeros has deviation sqrt(eps); rows of 1e18 have squares beyond binary32 only where a mean of squares does."""
    t, form = make(4, 400, torch.float32, seed=5, rate=0.0)
    t["y"][1] = 0.0
    t["x"][1] = 0.0
    t["x"][2] *= 1e17
    t["y"][3] *= 1e17
    check(t, form)


def test_weights_gradients_into_a_row_and_no_rows():
    t, form = make(64, 256, torch.bfloat16, seed=6, groups=2)
    s, z, stats, got = check(t, form)
    row = torch.full((3 + 256 + 512 + 256,), 7.0, device="cuda")
    post, gate, pre = row[1:257], row[257:769].view(2, 256), row[769:1025]
    bz.join_backward(t["x"], t["y"], stats, ds=t["ds"], dz=t["dz"], **form, dw_post=post, dgate=gate, dw_pre=pre)
    assert torch.equal(post, got["dw_post"]) and torch.equal(gate, got["dgate"]) and torch.equal(pre, got["dw_pre"])
    assert float(row[0]) == 7 and (row[1025:] == 7).all()
    none = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    s0, z0, stats0 = bz.join(none, none, **form)
    for value in bz.join_backward(none, none, stats0, ds=none, dz=none, **form)[2:]:
        assert (value == 0).all()


@pytest.mark.parametrize("n", [100, 4096, 12000])
def test_in_place_graph_and_other_stream(n):
    t, form = make(200, n, torch.bfloat16, seed=7)
    s, z, stats = bz.join(t["x"], t["y"], **form)
    want = bz.join_backward(t["x"], t["y"], stats, ds=t["ds"], dz=t["dz"], **form)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x, y, ds, dz = t["x"].clone(), t["y"].clone(), t["ds"].clone(), t["dz"].clone()
        got = bz.join(x, y, **form, s=x, z=y)
        back = bz.join_backward(t["x"], t["y"], stats, ds=ds, dz=dz, **form, dx=ds, dy=dz)
        y2 = t["y"].clone()
        own = bz.join_backward(t["x"], y2, stats, ds=t["ds"], dz=t["dz"], **form, dy=y2)
    side.synchronize()
    assert torch.equal(x, s) and torch.equal(y, z) and torch.equal(got[2], stats)
    assert all(torch.equal(a, b) for a, b in zip(back, want)) and all(torch.equal(a, b) for a, b in zip(own, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s2, z2, stats2 = bz.join(t["x"], t["y"], **form)
        back = bz.join_backward(t["x"], t["y"], stats2, ds=t["ds"], dz=t["dz"], **form)
    for _ in range(3):
        graph.replay()
    assert torch.equal(z2, z) and all(torch.equal(a, b) for a, b in zip(back, want))
    form["rng"].add_(1)
    graph.replay()
    fresh = bz.join(t["x"], t["y"], **form)
    assert torch.equal(z2, fresh[1]) and not torch.equal(z2, z)


def test_gradient_against_differences():
    t, form = make(4, 10, torch.float32, seed=8, groups=2, norm="layer", rate=0.2)
    s, z, stats = bz.join(t["x"], t["y"], **form, eps=EPS)
    got = dict(zip(("x", "y", "w_post", "gate", "w_pre"), bz.join_backward(t["x"], t["y"], stats, ds=t["ds"], dz=t["dz"], **form)))
    step = 1e-5

    def value(name, at, by):
        u, f = {k: v.cpu().double() if torch.is_tensor(v) else v for k, v in t.items()}, {k: v.cpu().double() if k in ("w_post", "gate", "w_pre") else v for k, v in form.items()}
        (u if name in u else f)[name][at] += by
        kind = f["norm"]
        a = normed(u["y"], kind)[0] * f["w_post"] * f["gate"].repeat_interleave(2, 0)
        keep = kept(form["rng"].tolist(), 40, 0.2).view(4, 10) * (65536 / (65536 - round(0.2 * 65536)))
        s = u["x"] + keep * a
        return float((s * u["ds"]).sum() + (normed(s, kind)[0] * f["w_pre"] * u["dz"]).sum())

    for name, at in (("x", (0, 3)), ("x", (3, 9)), ("y", (1, 1)), ("y", (2, 4)), ("w_post", (5,)), ("gate", (1, 7)), ("w_pre", (2,))):
        diff = (value(name, at, step) - value(name, at, -step)) / (2 * step)
        assert abs(diff - float(got[name][at])) < 2e-4, (name, at)
