"""The hybrid decoder with rows that are wider than the library's norm takes."""
import pytest
import torch

from paper_2502_18394_amd import binding, hybrid

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hkv,dtype", [(130, 13, torch.float32), (260, 26, torch.bfloat16)])
def test_wide_decoders(H, Hkv, dtype):
    print(f"case H={H} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    prompt, noise = torch.randint(0, 512, (40,), generator=g, device="cuda"), torch.rand((3, 2, 512), generator=g, device="cuda")
    sizes = dict(H=H, Hkv=Hkv, layers=2, window=256, page=16, dtype=dtype)
    a, ma = hybrid.run(prompt, 20, 2, 3, noise, captured=True, **sizes)
    b, mb = hybrid.run(prompt, 20, 2, 3, noise, captured=False, **sizes)
    assert ma.width * dtype.itemsize > binding.NORM_MOST_BYTES and torch.equal(a, b) and torch.equal(ma.pool.k_pages, mb.pool.k_pages)
    with pytest.raises(binding.SpectreError):                # such rows are still more than the call takes
        binding.add_norm(torch.zeros(1, ma.width, dtype=dtype, device="cuda"))
