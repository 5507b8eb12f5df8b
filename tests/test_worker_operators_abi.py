"""Refusals of the worker's operators: every call here returns from the host's checks, before anything is launched."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from paper_2010_04902_b200 import build as bz_build

BIG = 1 << 40
F = ctypes.c_void_p(256)      # never dereferenced
ODD = ctypes.c_void_p(257)
S = (ctypes.c_int64 * 3)(80, 40, 10)


@pytest.fixture(scope="module")
def L():
    bz_build.build()
    return bz.lib()


def test_glu(L):
    def call(x=F, ld_x=8, wg=F, wu=F, ld_w=8, m=4, n=6, k=8, dtype=bz.BF16, act=0, h=F, ld_h=6, preact=None, ws=None, size=0):
        return L.bz_glu(x, ld_x, wg, wu, ld_w, m, n, k, dtype, act, h, ld_h, preact, ws, size, None)

    n0 = bz.kernel_launch_count()
    for bad in (dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(ld_x=7), dict(ld_w=7), dict(ld_h=5), dict(m=-1), dict(n=-1),
                dict(k=-1), dict(dtype=3), dict(dtype=-1), dict(act=4), dict(act=-1), dict(x=ODD), dict(wu=ODD), dict(h=ODD),
                dict(preact=ctypes.c_void_p(264))):
        assert call(**bad) == bz.ERR_INVALID_ARG, bad
    for bad in (dict(dtype=bz.F32), dict(m=BIG), dict(n=BIG, ld_h=BIG), dict(k=BIG, ld_x=BIG, ld_w=BIG)):
        assert call(**bad) == bz.ERR_UNSUPPORTED, bad
    need = L.bz_glu_workspace_bytes(40, 6, 9, bz.BF16, 0)
    for ws, size in ((None, BIG), (F, need - 1), (ctypes.c_void_p(264), BIG)):      # operands that have to be laid out first
        assert call(m=40, k=9, ld_x=9, ld_w=9, ws=ws, size=size) == bz.ERR_WORKSPACE
    assert call(m=0) == bz.OK and call(n=0, wg=None, wu=None) == bz.OK
    assert bz.kernel_launch_count() == n0


def test_glu_backward(L):
    def call(x=F, ld_x=8, wg=F, wu=F, ld_w=8, preact=F, dh=F, ld_dh=6, m=4, n=6, k=8, dtype=bz.F16, act=0, dx=F, ld_dx=8, dwg=F, dwu=F, ld_dw=8,
             grad=bz.F16, ws=F, size=BIG):
        return L.bz_glu_backward(x, ld_x, wg, wu, ld_w, preact, dh, ld_dh, m, n, k, dtype, act, dx, ld_dx, dwg, dwu, ld_dw, grad, ws, size, None)

    n0 = bz.kernel_launch_count()
    for bad in (dict(x=None), dict(wg=None), dict(wu=None), dict(preact=None), dict(dh=None), dict(dwg=None), dict(dwu=None), dict(ld_dh=5),
                dict(ld_dx=7), dict(ld_dw=7), dict(ld_x=7), dict(ld_w=7), dict(grad=bz.BF16), dict(grad=9), dict(act=7), dict(m=-1),
                dict(dh=ODD), dict(dx=ODD), dict(dwg=ODD), dict(dx=None, dwg=None, dwu=None), dict(preact=ctypes.c_void_p(264)),
                dict(grad=bz.F32, dwg=ctypes.c_void_p(258))):
        assert call(**bad) == bz.ERR_INVALID_ARG, bad
    assert call(dtype=bz.F32, grad=bz.F32) == bz.ERR_UNSUPPORTED and call(m=BIG) == bz.ERR_UNSUPPORTED
    assert call(m=1 << 30, n=1 << 30, ld_dh=1 << 30) == bz.ERR_UNSUPPORTED
    need = L.bz_glu_workspace_bytes(4, 6, 8, bz.F16, 1)
    for ws, size in ((None, BIG), (F, need - 1), (ctypes.c_void_p(264), BIG)):
        assert call(ws=ws, size=size) == bz.ERR_WORKSPACE
    assert call(m=0, n=0) == bz.OK and call(k=0) == bz.OK
    assert bz.kernel_launch_count() == n0
    assert need > 0 and need % 256 == 0
    for args in ((-1, 6, 8, bz.F16, 1), (4, -1, 8, bz.F16, 1), (4, 6, -1, bz.F16, 1), (4, 6, 8, bz.F32, 1), (4, 6, 8, 5, 1)):
        assert L.bz_glu_workspace_bytes(*args) == 0


def test_bias_softmax(L):
    def both(scores=F, ss=S, dtype=bz.F16, b=1, h=2, tq=4, tk=10, table=F, buckets=32, distance=128, bi=1, causal=0, scale=1.0, probs=F, sp=S,
             stats=F, dprobs=F, sd=S, ds=F, so=S, dt=F, ws=F, size=BIG):
        head = (scores, ss, dtype, b, h, tq, tk, table, buckets, distance, bi, causal, scale, None, None)
        return (L.bz_bias_softmax(*head, probs, sp, stats, None),
                L.bz_bias_softmax_backward(*head, stats, dprobs, sd, ds, so, dt, ws, size, None))

    n0 = bz.kernel_launch_count()
    for bad in (dict(scores=None), dict(ss=None), dict(dtype=7), dict(b=-1), dict(h=-1), dict(tq=-1), dict(tk=-1), dict(table=None),
                dict(buckets=1), dict(buckets=33), dict(buckets=2), dict(distance=8), dict(scale=float("nan")), dict(scores=ODD),
                dict(stats=ctypes.c_void_p(260))):
        assert both(**bad) == (bz.ERR_INVALID_ARG, bz.ERR_INVALID_ARG), bad
    for bad in (dict(buckets=258), dict(distance=2049), dict(b=65536), dict(h=65536), dict(tq=1 << 31), dict(tk=1 << 31)):
        assert both(**bad) == (bz.ERR_UNSUPPORTED, bz.ERR_UNSUPPORTED), bad
    for bad in (dict(probs=None, stats=None), dict(sp=None, dprobs=None), dict(probs=ODD, sd=None), dict(probs=None, ds=None, dt=None),
                dict(probs=None, so=None), dict(probs=None, ds=ODD)):
        assert both(**bad) == (bz.ERR_INVALID_ARG, bz.ERR_INVALID_ARG), bad
    back = (ctypes.c_int64 * 3)(80, -40, 10)
    assert both(ss=back) == (bz.ERR_INVALID_ARG, bz.ERR_INVALID_ARG) and both(sp=back, sd=back) == (bz.ERR_INVALID_ARG, bz.ERR_INVALID_ARG)
    for bad in (dict(ws=None), dict(ws=ctypes.c_void_p(264)), dict(size=8)):
        assert both(probs=None, **bad)[1] == bz.ERR_WORKSPACE
    for none in (dict(b=0), dict(h=0), dict(tq=0), dict(tk=0)):
        assert both(dt=None, **none) == (bz.OK, bz.OK)
    assert bz.kernel_launch_count() == n0
    assert L.bz_bias_softmax_workspace_bytes(2, 3, 100, 100, 32) >= 2 * 3 * 32 * 4
    assert L.bz_bias_softmax_workspace_bytes(0, 3, 100, 100, 32) == 0 and L.bz_bias_softmax_workspace_bytes(2, 3, 100, 100, 1000) == 0


def test_distill(L):
    def both(logits=F, ld=10, dtype=bz.F16, m=4, v=10, teacher=F, index=F, t=3, T=1.0, dloss=None, loss=F, stats=F, d=F, ld_d=10):
        return (L.bz_distill(logits, ld, dtype, m, v, teacher, index, t, T, dloss, loss, stats, d, ld_d, None),
                L.bz_distill_backward(logits, ld, dtype, m, v, teacher, index, t, T, stats, dloss, d, ld_d, None))

    n0 = bz.kernel_launch_count()
    for bad in (dict(logits=None), dict(ld=9), dict(dtype=3), dict(m=-1), dict(v=-1), dict(teacher=None), dict(index=None), dict(t=0), dict(T=0.0),
                dict(T=-1.0), dict(T=float("inf")), dict(T=float("nan")), dict(ld_d=9), dict(logits=ODD), dict(d=ODD),
                dict(stats=ctypes.c_void_p(260)), dict(loss=None, stats=None, d=None)):
        assert both(**bad) == (bz.ERR_INVALID_ARG, bz.ERR_INVALID_ARG), bad
    assert L.bz_distill_backward(F, 10, bz.F16, 4, 10, F, F, 3, 1.0, None, None, F, 10, None) == bz.ERR_INVALID_ARG      # no stats
    for bad in (dict(v=1 << 31, ld=1 << 31, ld_d=1 << 31), dict(t=1025)):
        assert both(**bad) == (bz.ERR_UNSUPPORTED, bz.ERR_UNSUPPORTED), bad
    assert both(m=0, teacher=None, index=None, loss=None, stats=None, d=None) == (bz.OK, bz.OK)
    assert bz.kernel_launch_count() == n0


def test_python_side():
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        bz.glu(x.half(), x.half(), x.half())                      # not on the GPU
    with pytest.raises(ValueError):
        bz.glu(x, torch.zeros(3, 7), torch.zeros(3, 7))
    with pytest.raises(ValueError):
        bz.glu(x.expand(2, 4, 8), x, x)
    with pytest.raises(ValueError):
        bz.glu(torch.zeros(1, 8).expand(4, 8), x, x)              # rows that repeat have no leading dimension
    with pytest.raises(ValueError):
        bz.bias_softmax(torch.zeros(2, 3, 4), torch.zeros(32, 3))
    with pytest.raises(TypeError):
        bz.distill(torch.zeros(3, 9), torch.zeros(3, 2), torch.zeros(3, 2, dtype=torch.int32))


def test_bias_softmax_outputs_that_overlap(L):
    """Expanded and interleaved outputs: rows would overwrite one another."""
    three = lambda *s: (ctypes.c_int64 * 3)(*s)  # noqa: E731
    S2 = three(80, 40, 10)

    def both(out, b=2, h=2, tq=4, tk=10):
        head = (F, S2, bz.F16, b, h, tq, tk, F, 32, 128, 1, 0, 1.0, None, None)
        return (L.bz_bias_softmax(*head, F, out, None, None), L.bz_bias_softmax_backward(*head, F, F, S2, F, out, F, F, BIG, None))

    n0 = bz.kernel_launch_count()
    for out in (three(0, 40, 10), three(80, 0, 10), three(80, 40, 0), three(80, 40, 9), three(80, 39, 10), three(79, 40, 10), three(40, 40, 10),
                three(10, 20, 30), three(1 << 62, 1 << 62, 10)):
        assert both(out) == (bz.ERR_INVALID_ARG, bz.ERR_INVALID_ARG), list(out)
    # rows apart in any order, gaps, dimensions of one with any stride: past this check, refused for the workspace
    for out, n in ((three(80, 40, 10), {}), (three(40, 80, 10), {}), (three(10, 20, 40), {}), (three(1 << 62, 40, 10), {}), (three(100, 50, 11), {}),
                   (three(0, 0, 0), dict(b=1, h=1, tq=1)), (three(3, 10, 0), dict(b=1, h=3, tq=1))):
        assert both_backward(L, S2, out, **n) == bz.ERR_WORKSPACE, list(out)
    assert bz.kernel_launch_count() == n0


def both_backward(L, strides, out, b=2, h=2, tq=4, tk=10):
    return L.bz_bias_softmax_backward(F, strides, bz.F16, b, h, tq, tk, F, 32, 128, 1, 0, 1.0, None, None, F, F, strides, F, out, F, None, 0, None)


def test_glu_workspace_sizes(L):
    size = L.bz_glu_workspace_bytes
    assert size(1, 10922, 4096, bz.BF16, 0) == size(32, 7, 9, bz.F16, 0) == 0       # up to 32 rows nothing is laid out
    assert size(33, 7, 9, bz.F16, 0) >= 2 * (33 + 2 * 7) * 9 and size(1, 7, 9, bz.F16, 1) > 0
    most = (1 << 31) - 512
    assert size(40, 8, most, bz.BF16, 0) > 0
    for m, n, k in ((most + 1, 8, 8), (40, most + 1, 8), (40, 8, most + 1), (BIG, 8, 8)):
        assert size(m, n, k, bz.BF16, 0) == size(m, n, k, bz.BF16, 1) == 0
    assert size(1 << 20, 1 << 19, 8, bz.BF16, 1) == 0 and size(1 << 20, (1 << 19) - 8, 8, bz.BF16, 1) > 0


def test_bias_softmax_workspace_of_many_heads_and_queries(L):
    """The size takes no longer for more heads and queries (it had counted rounds of CTAs one by one: hours at the limits),
    and it does not wrap."""
    ask = ("import sys; sys.path.insert(0, %r)\nfrom paper_2010_04902_b200 import binding as bz\nf = bz.lib().bz_bias_softmax_workspace_bytes\n"
           "print(f(65535, 65535, 2 ** 31 - 1, 1, 256), f(512, 512, 512, 1, 32), f(1, 1, 1, 1 << 31, 32))" % os.path.dirname(os.path.dirname(__file__)))
    r = subprocess.run([sys.executable, "-c", ask], capture_output=True, text=True, timeout=60)
    largest, usual, refused = (int(v) for v in r.stdout.split())
    assert largest == 2 ** 64 - 256 and refused == 0
    assert 512 * 512 * 8 * 32 * 4 <= usual <= 2 * 512 * 512 * 8 * 32 * 4      # eight chunks of 64 queries a head


def test_glu_enqueues_nothing_when_a_tensor_map_cannot_be_made():
    """Where there is no driver no map can be made: operands off the 16-byte grid (which are copied first) and the backward
    call (whose first kernel comes before the products) must have launched nothing.  No device is visible to the process."""
    try:
        ctypes.CDLL("libcuda.so.1")
        pytest.skip("there is a driver")
    except OSError:
        pass
    ask = """if 1:
        import sys; sys.path.insert(0, %r)
        import ctypes
        from paper_2010_04902_b200 import binding as bz
        P = ctypes.c_void_p(256)
        a = bz.lib().bz_glu(P, 9, P, P, 9, 40, 6, 9, bz.BF16, 0, P, 6, None, P, 1 << 40, None)
        b = bz.lib().bz_glu_backward(P, 8, P, P, 8, P, P, 6, 40, 6, 8, bz.BF16, 0, P, 8, P, P, 8, bz.BF16, P, 1 << 40, None)
        print(a, b, bz.kernel_launch_count())
    """ % os.path.dirname(os.path.dirname(__file__))
    r = subprocess.run([sys.executable, "-c", ask], capture_output=True, text=True, timeout=120, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
    assert r.stdout.split() == [str(bz.ERR_UNSUPPORTED)] * 2 + ["0"], r.stdout + r.stderr[-1000:]


def test_tensors_that_require_a_gradient():
    """Refused while gradients are recorded; otherwise the calls go on (here to the refusal of tensors that are not on a GPU)."""
    x, w, table = torch.zeros(4, 8).half(), torch.zeros(3, 8).half(), torch.zeros(32, 2)
    scores, teacher, index = torch.zeros(1, 2, 3, 4), torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32)
    g = lambda t: t.clone().requires_grad_(True)  # noqa: E731
    calls = [lambda: bz.glu(g(x), w, w), lambda: bz.glu(x, g(w), w), lambda: bz.glu(x, w, g(w)), lambda: bz.bias_softmax(g(scores), table),
             lambda: bz.bias_softmax(scores, g(table)), lambda: bz.distill(g(x), teacher, index)]
    for call in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(TypeError):
            call()


def test_distill_temperatures_without_an_inverse(L):
    """Below 4.3e-39 logits / T cannot be formed in binary32: every loss would be NaN."""
    S1 = (F, 10, bz.F16, 4, 10, F, F, 3)
    n0 = bz.kernel_launch_count()
    for T in (1e-39, 4.2e-39, 2.0 ** -149):
        assert L.bz_distill(*S1, T, None, F, F, F, 10, None) == bz.ERR_INVALID_ARG
        assert L.bz_distill_backward(*S1, T, F, None, F, 10, None) == bz.ERR_INVALID_ARG
    for T in (4.3e-39, 3.4028235e38):     # past this check: the loss and its gradient have nowhere to go
        assert L.bz_distill(*S1, T, None, None, None, None, 10, None) == bz.ERR_INVALID_ARG
        assert L.bz_distill(F, 9, bz.F16, 0, 10, F, F, 3, T, None, F, F, F, 10, None) == bz.OK
    assert bz.kernel_launch_count() == n0
