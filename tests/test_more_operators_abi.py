"""Refusals of the token losses, dropout and the join: every call here returns from the host's checks, before anything is
launched."""
import ctypes
import math

import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from paper_2010_04902_b200 import build as bz_build

BIG = 1 << 40
F = ctypes.c_void_p(256)      # never dereferenced
ODD = ctypes.c_void_p(257)
EIGHT = ctypes.c_void_p(264)
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def L():
    bz_build.build()
    return bz.lib()


def test_policy(L):
    def call(logits=F, ld=10, dtype=bz.F16, m=4, v=10, index=F, old=F, ref=F, adv=F, T=1.0, lo=0.2, hi=0.2, kl=0.1, dloss=None, loss=F, logp=F, stats=F,
             d=F, ld_d=10):
        return L.bz_policy(logits, ld, dtype, m, v, index, old, ref, adv, T, lo, hi, kl, dloss, loss, logp, stats, d, ld_d, None)

    n0 = bz.kernel_launch_count()
    for bad in (dict(logits=None), dict(ld=9), dict(dtype=3), dict(m=-1), dict(v=-1), dict(index=None), dict(adv=None), dict(ref=None), dict(T=0.0), dict(T=-1.0),
                dict(T=INF), dict(T=NAN), dict(T=4.2e-39), dict(lo=-0.1), dict(lo=1.1), dict(lo=NAN), dict(hi=-0.1), dict(hi=NAN), dict(kl=-0.1), dict(kl=INF),
                dict(kl=NAN), dict(ld_d=9), dict(logits=ODD), dict(d=ODD), dict(stats=EIGHT), dict(loss=None, logp=None, stats=None, d=None),
                dict(index=ODD), dict(old=ODD), dict(ref=ODD), dict(adv=ODD), dict(dloss=ODD), dict(loss=ODD), dict(logp=ODD)):
        assert call(**bad) == bz.ERR_INVALID_ARG, bad
    for bad in (dict(v=1 << 31, ld=1 << 31, ld_d=1 << 31), dict(v=(1 << 31) - 16383, ld=1 << 33, ld_d=1 << 33), dict(m=1 << 31), dict(ld=1 << 31), dict(ld_d=1 << 31)):
        assert call(**bad) == bz.ERR_UNSUPPORTED, bad
    assert call(m=0, index=None, adv=None, ref=None) == bz.OK
    assert bz.kernel_launch_count() == n0


def test_preference(L):
    def call(logits=F, ld=10, dtype=bz.F16, m=4, v=10, index=F, ref=F, starts=F, pairs=1, T=1.0, beta=0.1, margin=0.0, eps=0.0, mean=0, dloss=None, loss=F,
             reward=F, logp=F, stats=F, d=F, ld_d=10):
        return L.bz_preference(logits, ld, dtype, m, v, index, ref, starts, pairs, T, beta, margin, eps, mean, dloss, loss, reward, logp, stats, d, ld_d, None)

    n0 = bz.kernel_launch_count()
    for bad in (dict(logits=None), dict(ld=9), dict(dtype=-1), dict(m=-1), dict(v=-1), dict(index=None), dict(starts=None), dict(pairs=-1), dict(T=0.0), dict(T=NAN),
                dict(beta=NAN), dict(beta=INF), dict(margin=INF), dict(margin=NAN), dict(eps=-0.1), dict(eps=1.1), dict(eps=NAN), dict(stats=None), dict(logp=None), dict(stats=EIGHT),
                dict(ld_d=9), dict(d=ODD), dict(logits=ODD), dict(index=ODD), dict(starts=ODD), dict(ref=ODD), dict(dloss=ODD), dict(loss=ODD), dict(reward=ODD), dict(logp=ODD)):
        assert call(**bad) == bz.ERR_INVALID_ARG, bad
    for bad in (dict(v=1 << 31, ld=1 << 31, ld_d=1 << 31), dict(v=(1 << 31) - 16383, ld=1 << 33, ld_d=1 << 33), dict(m=1 << 31), dict(pairs=1 << 30)):
        assert call(**bad) == bz.ERR_UNSUPPORTED, bad
    assert call(m=0, pairs=0, starts=None, stats=None) == bz.OK
    assert bz.kernel_launch_count() == n0


def test_token_loss_backward(L):
    def call(logits=F, ld=10, dtype=bz.F32, m=4, v=10, index=F, T=1.0, stats=F, dloss=None, places=0, d=F, ld_d=10):
        return L.bz_token_loss_backward(logits, ld, dtype, m, v, index, T, stats, dloss, places, d, ld_d, None)

    n0 = bz.kernel_launch_count()
    for bad in (dict(logits=None), dict(ld=9), dict(dtype=9), dict(m=-1), dict(index=None), dict(T=0.0), dict(stats=None), dict(stats=EIGHT), dict(d=None), dict(ld_d=9),
                dict(logits=ODD), dict(d=ODD), dict(index=ODD), dict(dloss=ODD), dict(dloss=F, places=-1)):
        assert call(**bad) == bz.ERR_INVALID_ARG, bad
    assert call(m=1 << 31) == bz.ERR_UNSUPPORTED
    assert call(m=0) == bz.OK and call(v=0) == bz.OK
    assert bz.kernel_launch_count() == n0


def test_dropout(L):
    def call(x=F, ld=10, dtype=bz.F16, m=4, n=10, rate=0.1, rng=F, out=F, ld_out=10):
        return L.bz_dropout(x, ld, dtype, m, n, rate, rng, out, ld_out, None)

    n0 = bz.kernel_launch_count()
    for bad in (dict(x=None), dict(out=None), dict(rng=None), dict(rng=ctypes.c_void_p(260)), dict(ld=9), dict(ld_out=9), dict(dtype=3), dict(m=-1), dict(n=-1),
                dict(rate=-0.1), dict(rate=1.0), dict(rate=0.999999), dict(rate=NAN), dict(x=ODD), dict(out=ODD)):
        assert call(**bad) == bz.ERR_INVALID_ARG, bad
    for bad in (dict(m=BIG), dict(n=BIG, ld=BIG, ld_out=BIG), dict(m=1 << 30, n=1 << 20, ld=1 << 20, ld_out=1 << 20), dict(ld=BIG)):
        assert call(**bad) == bz.ERR_UNSUPPORTED, bad
    assert call(m=0, x=None, rng=None) == bz.OK and call(n=0) == bz.OK
    assert bz.kernel_launch_count() == n0


def test_join(L):
    def both(x=F, ld=10, y=F, dtype=bz.F16, m=4, n=10, norm=0, eps=1e-6, post=F, gate=F, groups=2, rs=1.0, bs=1.0, rate=0.1, rng=F, pre=F, e=F, f=F, ld_e=10, stats=F,
             ds=F, dz=F, dpost=F, dgate=F, dpre=F, ws=F, size=BIG, which="both"):
        # a call that one of the two accepts is made of the other alone
        return (which != "backward" and L.bz_join(x, ld, y, ld, dtype, m, n, norm, eps, post, gate, groups, rs, bs, rate, rng, pre, e, ld_e, f, ld_e, stats, None),
                which != "forward" and L.bz_join_backward(x, ld, y, ld, dtype, m, n, norm, post, gate, groups, rs, bs, rate, rng, pre, stats, ds, ld, dz, ld, e, ld_e, f, ld_e, dpost, dgate, dpre,
                                   ws, size, None))

    n0 = bz.kernel_launch_count()
    two = (bz.ERR_INVALID_ARG, bz.ERR_INVALID_ARG)
    for bad in (dict(x=None), dict(ld=9), dict(dtype=3), dict(m=-1), dict(n=-1), dict(norm=2), dict(norm=-1), dict(groups=-1), dict(groups=0), dict(groups=3), dict(gate=None),
                dict(rs=NAN), dict(rs=INF), dict(bs=NAN), dict(rate=1.0), dict(rate=-0.1), dict(rng=None), dict(rng=ctypes.c_void_p(260)), dict(y=None), dict(x=ODD), dict(y=ODD),
                dict(e=ODD), dict(f=ODD), dict(ld_e=9), dict(stats=EIGHT), dict(post=ODD), dict(gate=ODD), dict(pre=ODD)):
        assert both(**bad) == two, bad
    for bad in (dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(e=None, f=None), dict(f=None), dict(pre=None)):     # no output; z without w_pre or the reverse
        assert both(**bad, which="forward")[0] == bz.ERR_INVALID_ARG, bad
    for bad in (dict(post=None, stats=None), dict(stats=None), dict(post=None), dict(gate=None, groups=0), dict(pre=None, dpre=None), dict(pre=None, dz=None),
                dict(e=None, f=None, dpost=None, dgate=None, dpre=None)):
        assert both(**bad, which="backward")[1] == bz.ERR_INVALID_ARG, bad
    for bad in (dict(m=1 << 31, groups=1), dict(n=16385, ld=20000, ld_e=20000), dict(ld=1 << 31), dict(ld_e=1 << 31)):
        assert both(**bad) == (bz.ERR_UNSUPPORTED, bz.ERR_UNSUPPORTED), bad
    need = L.bz_join_workspace_bytes(4, 10, 2)
    for bad in (dict(ws=None), dict(ws=EIGHT), dict(size=need - 1)):
        assert both(**bad, which="backward")[1] == bz.ERR_WORKSPACE
    assert both(n=0) == (bz.OK, bz.OK) and both(m=0, dpost=None, dgate=None, dpre=None) == (bz.OK, bz.OK)
    assert bz.kernel_launch_count() == n0
    assert need > 0 and need % 256 == 0
    for args in ((-1, 10, 0), (4, -1, 0), (4, 10, -1), (4, 10, 3), (4, 16385, 0), (1 << 31, 10, 0)):
        assert L.bz_join_workspace_bytes(*args) == 0


def test_python_side():
    x, i32 = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        bz.policy(x, i32, torch.zeros(4))                          # not on the GPU
    with pytest.raises(ValueError):
        bz.policy(x.t(), i32, torch.zeros(8))
    with pytest.raises(ValueError):
        bz.preference(torch.zeros(1, 8).expand(4, 8), i32, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        bz.token_loss_backward(x, i32, torch.zeros(4, 4))
    with pytest.raises(TypeError):
        bz.dropout(x, 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError):
        bz.join(x, x)
    with pytest.raises(ValueError):
        bz.join(x[0], x[0])
    with pytest.raises(TypeError):
        bz.join_backward(x, x, torch.zeros(4, 4))


def test_tensors_that_require_a_gradient():
    """Refused while gradients are recorded; otherwise the calls go on (here to the refusal of tensors that are not on a GPU)."""
    x, index, w = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(8)
    g = lambda t: t.clone().requires_grad_(True)  # noqa: E731
    rng, starts = torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: bz.policy(g(x), index, w[:4]), lambda: bz.preference(g(x), index, starts), lambda: bz.dropout(g(x), 0.1, rng), lambda: bz.join(g(x), x),
                 lambda: bz.join(x, g(x)), lambda: bz.join(x, x, w_post=g(w)), lambda: bz.join(x, x, gate=g(w)[None]), lambda: bz.join(x, x, w_pre=g(w))):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(TypeError):
            call()


def test_workspace_of_many_groups(L):
    """A part each once there are many groups: dgate needs no sums then, and the bytes do not grow with them."""
    size = L.bz_join_workspace_bytes
    assert 0 < size(1 << 20, 1024, 1 << 20) < size(1 << 20, 1024, 1) == size(1 << 20, 1024, 0)
    assert size(1 << 20, 1024, 1 << 19) == size(1 << 20, 1024, 1 << 20)
