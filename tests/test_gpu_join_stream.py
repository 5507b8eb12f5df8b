"""join_backward() takes the stream that went into join() or the one that came out of it: both are [m][n] of one type, and the call
reads the one that its stats keep."""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from test_gpu_join import EPS, check, make

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def all_equal(a, b):
    return all((p is None and q is None) or torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,pad,norm,post,rate", [(1, 64, 0, "rms", True, 0.0), (777, 1001, 3, "layer", True, 0.1), (300, 4096, 0, "rms", True, 0.1),
                                                    (40, 300, 0, "rms", False, 0.25), (9, 9000, 0, "layer", False, 0.0)])
def test_either_stream(m, n, pad, norm, post, rate, dtype):
    t, form = make(m, n, dtype, seed=n, pad=pad, norm=norm, post=post, rate=rate, residual=1.7, scale=0.5)
    s, _, stats, want = check(t, form)         # from x, against 64 bits
    want = tuple(want.values())
    for stream in (s, s.clone(), t["x"].clone()):
        assert all_equal(bz.join_backward(stream, t["y"], stats, ds=t["ds"], dz=t["dz"], **form), want)
    for stream in (t["x"], t["x"].clone()):
        assert all_equal(bz.join_backward(x=stream, y=t["y"], stats=stats, ds=t["ds"], dz=t["dz"], **form), want)
        # numbers alone keep no stream: x it is
        assert all_equal(bz.join_backward(stream, t["y"], stats.clone(), ds=t["ds"], dz=t["dz"], **form), want)


def test_a_stream_that_was_written_since():
    t, form = make(20, 128, torch.bfloat16, seed=1)
    s, _, stats = bz.join(t["x"], t["y"], **form)
    want = bz.join_backward(s, t["y"], stats, ds=t["ds"], dz=t["dz"], **form)
    x = t["x"].clone()
    t["x"].add_(1.0)
    with pytest.raises(ValueError, match="written"):
        bz.join_backward(s, t["y"], stats, ds=t["ds"], dz=t["dz"], **form)
    assert all_equal(bz.join_backward(x=x, y=t["y"], stats=stats, ds=t["ds"], dz=t["dz"], **form), want)
    # these calls' own writes count as well
    form0 = dict(form, w_post=None, gate=None, w_pre=None, rate=0.0, rng=None)
    for write in (lambda a: bz.join(t["y"], t["y"], **form0, s=a), lambda a: bz.join(t["y"], w_pre=form["w_pre"], z=a), lambda a: bz.dropout(a, 0.5, form["rng"], out=a),
                  lambda a: bz.join_backward(x, t["y"], stats, ds=t["ds"], dz=t["dz"], **form, dx=a), lambda a: bz.join_backward(x=x, y=t["y"], stats=stats, ds=t["ds"], dz=t["dz"], **form, dy=a)):
        old = x.clone()
        s, _, stats = bz.join(old, t["y"], **form)
        write(old)
        with pytest.raises(ValueError, match="written"):
            bz.join_backward(s, t["y"], stats, ds=t["ds"], dz=t["dz"], **form)
    # the other half of a buffer may be written: the same memory is taken as it is
    buffer = torch.stack([x, x])
    _, _, stats = bz.join(buffer[0], t["y"], **form)
    buffer[1].zero_()
    assert all_equal(bz.join_backward(buffer[0], t["y"], stats, ds=t["ds"], dz=t["dz"], **form), want)


def test_a_result_written_over_x():
    t, form = make(20, 128, torch.bfloat16, seed=1)
    x, y = t["x"].clone(), t["y"]
    _, _, stats0 = bz.join(x, y, **form)
    want = bz.join_backward(x, y, stats0, ds=t["ds"], dz=t["dz"], **form)
    for over in ("s", "z"):
        x = t["x"].clone()
        stats = bz.join(x, y, **form, **{over: x})[2]
        with pytest.raises(ValueError, match="written"):
            bz.join_backward(x, y, stats, ds=t["ds"], dz=t["dz"], **form)
        assert all_equal(bz.join_backward(t["x"], y, stats, ds=t["ds"], dz=t["dz"], **form), want)


def test_other_shapes_are_refused():
    t, form = make(20, 128, torch.bfloat16, seed=1)
    _, _, stats = bz.join(t["x"], t["y"], **form)
    for stream in (t["x"][:10], t["x"].float(), t["x"].cpu()):
        with pytest.raises((ValueError, TypeError)):
            bz.join_backward(stream, t["y"], stats, ds=t["ds"], dz=t["dz"], **form)


def test_captured_and_replayed():
    t, form = make(50, 256, torch.bfloat16, seed=3)
    bz.join(t["x"], t["y"], **form)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s, _, stats = bz.join(t["x"], t["y"], **form, eps=EPS)
        back = bz.join_backward(s, t["y"], stats, ds=t["ds"], dz=t["dz"], **form)
    t["x"].normal_()
    graph.replay()
    _, _, stats = bz.join(t["x"], t["y"], **form, eps=EPS)
    assert all_equal(back, bz.join_backward(t["x"], t["y"], stats, ds=t["ds"], dz=t["dz"], **form))


def test_tensors_of_inference_mode():
    """They count no writes."""
    t, form = make(20, 128, torch.bfloat16, seed=1)
    _, _, stats = bz.join(t["x"], t["y"], **form)
    want = bz.join_backward(t["x"], t["y"], stats, ds=t["ds"], dz=t["dz"], **form)
    with torch.inference_mode():
        x = t["x"].clone()
        s, _, stats = bz.join(x, t["y"], **form)
        assert all_equal(bz.join_backward(s, t["y"], stats, ds=t["ds"], dz=t["dz"], **form), want)
