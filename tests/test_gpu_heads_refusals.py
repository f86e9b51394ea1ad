"""Calls on heads that the library refuses, as the binding's caller sees them: the same error from all three calls, and nothing is written."""
import pytest
import torch

from paper_2502_18394_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("missing", ["wq", "wk"])
def test_one_weight_alone(missing):
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn(3, n, 64, generator=g).to(torch.bfloat16).cuda() for n in (4, 2))
    w = dict(wq=torch.ones(64, device="cuda"), wk=torch.ones(64, device="cuda"))
    w[missing] = None
    pool = binding.KvPages.empty(1, 4, 2, 64, 16, 1, 4)
    one = torch.tensor([0], dtype=torch.int32, device="cuda")
    pool.reserve(one, one + 3)
    out = torch.full_like(q, 7)
    calls = (lambda: binding.qk_norm_rotate(q, k, **w, q_out=out), lambda: binding.qk_norm_rotate_backward(q, k, q, k, **w),
             lambda: pool.append(0, q, k, k, torch.tensor([0, 3], dtype=torch.int32, device="cuda"), q_out=out, **w))
    for call in calls:
        with pytest.raises(binding.SpectreError, match="one of wq and wk is null"):
            call()
    assert (out == 7).all() and not pool.k_pages.any()
