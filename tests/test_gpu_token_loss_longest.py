"""Rows beyond what a cluster's shared memory holds (430 000 columns of binary32, 860 000 of 16 bits), read twice in whole words.
Tolerances as in test_gpu_token_loss."""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz
from test_gpu_token_loss import check_policy, check_preference, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,v,pad", [(torch.float32, 450001, 0), (torch.float32, 450000, 4), (torch.bfloat16, 900001, 0), (torch.float16, 900001, 3)])
def test_longest_rows(dtype, v, pad):
    x = make(5, v, dtype, v, pad)
    x["index"][:4] = torch.tensor([0, v - 1, -1, v // 2], dtype=torch.int32)
    d = check_policy(x)[3]
    form = {"old_logp": x["old"], "ref_logp": x["ref"], "kl": 0.05, "clip_low": 0.2, "clip_high": 0.28}
    own = x["logits"].clone() if pad == 0 else torch.empty(5, v + pad, dtype=dtype, device="cuda")[:, :v].copy_(x["logits"])
    bz.policy(own, x["index"], x["adv"], **form, dloss=x["dloss"], dlogits=own)
    assert torch.equal(own, d)
    want = check_preference(x, [0, 2, 4])[4]
    own.copy_(x["logits"])
    starts = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    bz.preference(own, x["index"], starts, ref_logp=x["ref"], dloss=x["dloss"][:1].contiguous(), dlogits=own)
    assert torch.equal(own, want)
