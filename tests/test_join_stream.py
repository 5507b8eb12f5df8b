"""Which stream join_backward() reads: the host's side, without a GPU."""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz


def kept(x, over=False):
    """Stats as join() returns them."""
    stats = torch.zeros(x.shape[0], 4)
    stats._stream_in = x, x._version, over
    return stats


def test_the_stream_that_stats_keep():
    x = torch.randn(4, 8)
    s, stats = x + 1, kept(x)
    for stream in (x, s, x.clone()):
        assert bz._stream_in(stream, stats) is x
    other = torch.randn(4, 8)
    assert bz._stream_in(other, stats.clone()) is other         # a copy of the numbers keeps nothing
    for wrong in (torch.zeros(3, 8), torch.zeros(4, 8, dtype=torch.float16), torch.zeros(4, 8, device="meta")):
        with pytest.raises(ValueError, match="like the x"):
            bz._stream_in(wrong, stats)


def test_written_since():
    x = torch.randn(2, 4, 8)
    stats, s = kept(x[0]), x[0] + 1
    x[1].zero_()                                                  # counted as a write to x[0] too: the same memory is taken as it is
    assert bz._stream_in(x[0], stats).data_ptr() == x.data_ptr()
    with pytest.raises(ValueError, match="written since"):
        bz._stream_in(s, stats)


def test_s_over_x():
    x = torch.randn(4, 8)
    before = x.clone()
    stats = kept(x, over=True)
    with pytest.raises(ValueError, match="written over its x"):
        bz._stream_in(x, stats)
    assert bz._stream_in(before, stats) is before


def test_arguments():
    x, stats = torch.zeros(4, 8), torch.zeros(4, 4)
    for call in (lambda: bz.join_backward(x, x), lambda: bz.join_backward(y=x, stats=stats), lambda: bz.join_backward(x, x, stats, x=x)):
        with pytest.raises(TypeError, match="needs stats"):
            call()
    with pytest.raises(TypeError, match="CUDA"):
        bz.join_backward(x=x, y=x, stats=stats)
