"""Workspaces that calls do not take (no device is touched)."""
import pytest
import torch

from paper_2502_18394_amd import binding


@pytest.mark.parametrize("ws", [torch.empty(4096, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8).expand(4096)])
def test_workspaces_in_host_memory(ws):
    """Kernels would write to an address that is not the device's."""
    with pytest.raises(ValueError, match="ws must be a contiguous device tensor"):
        binding._given(ws)
    with pytest.raises(ValueError, match="ws must be a contiguous device tensor"):
        binding._workspace(1024, "cpu", ws)
