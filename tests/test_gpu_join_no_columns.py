"""Joins of rows without columns do nothing, whatever takes part: empty tensors have no address."""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz


@pytest.mark.gpu
@pytest.mark.parametrize("m", [0, 1, 6])
def test_no_columns(m):
    x, w = torch.empty(m, 0, device="cuda"), torch.empty(0, device="cuda")
    form = {"w_post": w, "gate": torch.empty(1, 0, device="cuda"), "w_pre": w, "rate": 0.1, "rng": torch.tensor([1, 2], device="cuda")}
    s, z, stats = bz.join(x, x, **form)
    assert s.shape == z.shape == (m, 0)
    for got, like in zip(bz.join_backward(x, x, stats, ds=x, dz=x, **form), (x, x, w, form["gate"], w)):
        assert got.shape == like.shape
