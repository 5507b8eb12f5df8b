"""The tensor-core kernels of the gated block when a bounded wait runs out: one CTA of each pair stops loading after two
blocks of the contraction, so the other runs ahead by a ring, every wait ends after about a second, what is in flight is waited
for, and the kernels return.  The calls after that give the same bits as before."""
import time

import pytest
import torch

from paper_2010_04902_b200 import binding as bz

pytestmark = [pytest.mark.gpu, pytest.mark.expired_waits]


@pytest.mark.parametrize("which", [1, 2])
@pytest.mark.parametrize("m,n,k", [(300, 500, 1024), (2000, 4096, 2048)])
def test_expired_waits_return_and_leave_nothing_behind(m, n, k, which):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(m, k, generator=g, device="cuda").to(torch.bfloat16)
    wg, wu = (torch.randn(n, k, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    dh = torch.randn(m, n, generator=g, device="cuda").to(torch.bfloat16)
    preact = torch.empty(2, m, n, device="cuda")

    def step():
        return (bz.glu(x, wg, wu, preact=preact),) + bz.glu_backward(x, wg, wu, preact, dh)

    want = step()
    torch.cuda.synchronize()
    before, t0 = bz.pipeline_timeouts(), time.time()
    bz.debug_stall_pipeline(which)
    try:
        step()
        torch.cuda.synchronize()
    finally:
        bz.debug_stall_pipeline(0)
    assert bz.pipeline_timeouts() > before and time.time() - t0 < 20
    counted = bz.pipeline_timeouts()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
    assert bz.pipeline_timeouts() == counted
