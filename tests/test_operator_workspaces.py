"""CPU checks: a workspace whose elements do not lie one behind the other is refused, since its size says nothing of its memory then."""
import pytest


def test_workspaces_that_are_not_contiguous(monkeypatch):
    import torch
    from paper_2407_08330_amd import binding

    class Device(torch.Tensor):  # a host tensor that says it is a device one (and is never used)
        is_cuda = True

    def device(t):
        return t.as_subclass(Device)
    binding._check_workspace(None)
    binding._check_workspace(device(torch.zeros(64, dtype=torch.uint8)))
    for t in (torch.zeros(1, dtype=torch.uint8).expand(1 << 30), torch.zeros(64, dtype=torch.uint8)[::2], torch.zeros(8, 8).t()):
        with pytest.raises(ValueError, match="workspace"):
            binding._check_workspace(device(t))
    with pytest.raises(ValueError, match="workspace"):
        binding._check_workspace(torch.zeros(64, dtype=torch.uint8))
