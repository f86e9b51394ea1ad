"""The norm's backward pass without a weight on the GPU: gradients of the rows are those of a weight of ones, bit for bit, however many workgroups have them."""
import pytest
import torch

from paper_2502_18394_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D", [(1, 64), (2, 1024), (31, 1024), (32, 1024), (33, 1024), (8, 2048), (9, 2048), (3, 4096), (8, 8192), (2, 7992), (0, 64), (1030, 128)])
def test_backward_without_a_weight(T, D, dtype):
    print(f"case T={T} D={D} {dtype}", flush=True)
    g = torch.Generator().manual_seed(T + D)
    total, dy, dsum = (torch.randn(T, D, generator=g).to(dtype).cuda() for _ in range(3))
    for e in (dsum, None):
        want, _ = binding.add_norm_backward(dy, total, torch.ones(D, device="cuda"), e, 1e-5)
        got, gw = binding.add_norm_backward(dy, total, None, e, 1e-5)
        assert gw is None and torch.equal(got, want)
