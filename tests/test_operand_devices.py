"""Tensors of one call on two devices: the fine-tuning calls refuse them before a kernel could read memory that it has no access to.
Devices are stood in for."""
import pytest
import torch

from paper_2010_04902_b200 import binding as bz


class On:
    """What the check looks at of a tensor."""

    def __init__(self, device):
        self.index, self.is_cuda = device, device >= 0
        self.device = "cuda:%d" % device if device >= 0 else "cpu"

    def get_device(self):
        return self.index


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)


def test_all_of_a_call_on_the_current_device():
    bz._here(On(0), "x", (On(0), None, On(0)))
    bz._here(On(0), "x", (On(-1),))            # the host's memory is the next check's business
    bz._here(On(-1), "x", (On(1),))
    with pytest.raises(ValueError, match="current device"):
        bz._here(On(1), "x", (On(1),))
    with pytest.raises(ValueError, match="another tensor of the call on cuda:1"):
        bz._here(On(0), "x", (None, On(0), On(1)))


class Stop(Exception):
    pass


def test_every_operand_is_looked_at(monkeypatch):
    """Each call hands all its tensors to the check."""
    seen = []

    def look(t, name, others=()):
        seen.extend([t, *others])
        raise Stop

    monkeypatch.setattr(bz, "_here", look)
    monkeypatch.setattr(bz, "_dtype", lambda t, name: bz.F32)
    monkeypatch.setattr(bz, "_packed", lambda t, shape, dtype, name: 0)
    t = lambda *shape: torch.zeros(shape)  # noqa: E731
    one = {"logits": t(4, 8), "index": t(4), "dloss": t(4), "dlogits": t(4, 8), "stats": t(4, 4)}
    both = {**one, "ref_logp": t(4), "loss": t(4), "logp": t(4)}
    form = {"w_post": t(8), "gate": t(1, 8), "w_pre": t(8), "rng": t(2), "stats": t(4, 4)}
    for call, given in ((bz.policy, {**both, "advantage": t(4), "old_logp": t(4)}), (bz.preference, {**both, "starts": t(3), "reward": t(2)}), (bz.token_loss_backward, one),
                        (bz.dropout, {"x": t(4, 8), "rng": t(2), "out": t(4, 8)}), (bz.join, {**form, "x": t(4, 8), "y": t(4, 8), "s": t(4, 8), "z": t(4, 8)}),
                        (bz.join_backward, {**form, **{k: t(4, 8) for k in ("x", "y", "ds", "dz", "dx", "dy")}, "dw_post": t(8), "dgate": t(1, 8), "dw_pre": t(8), "workspace": t(9)})):
        seen.clear()
        with pytest.raises(Stop):
            call(**given, **({"rate": 0.1} if "rng" in given else {}))
        assert {id(v) for v in given.values()} == {id(v) for v in seen if v is not None}
