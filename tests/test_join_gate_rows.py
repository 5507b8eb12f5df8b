"""A gate without rows."""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz


def test_a_gate_without_rows_is_no_gate_at_all():
    """It has no address, as none has: the call went on as if there were none."""
    with pytest.raises(ValueError, match="one group"):
        bz._join_form(4, 8, None, torch.empty(0, 8), None, 0.0, None)
    for shape in ((2, 7), (8,), (1, 2, 8)):
        with pytest.raises(ValueError, match="gate must be"):
            bz._join_form(4, 8, None, torch.empty(shape), None, 0.0, None)


@pytest.mark.gpu
def test_refused_by_both_calls():
    x = torch.randn(4, 8, device="cuda")
    gate = torch.empty(0, 8, device="cuda")
    with pytest.raises(ValueError, match="one group"):
        bz.join(x, x, gate=gate)
    stats = bz.join(x, x)[2]
    with pytest.raises(ValueError, match="one group"):
        bz.join_backward(x, x, stats, ds=x, gate=gate)
    # no rows: a gate of none fits them
    none = torch.empty(0, 8, device="cuda")
    s, _, stats = bz.join(none, none, gate=gate)
    assert s.shape == (0, 8) and bz.join_backward(none, none, stats, ds=none, gate=gate)[3].shape == (0, 8)
