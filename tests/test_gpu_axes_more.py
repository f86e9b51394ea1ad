"""Rotation whose pairs leave out the last axes of the positions, on the GPU: the same bits as with the rows that are read."""
import pytest
import torch

from paper_2502_18394_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("used", [1, 2, 3])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_positions_of_axes_that_no_pair_goes_by(d, used, dtype):
    print(f"case d={d} used={used} {dtype}", flush=True)
    g = torch.Generator().manual_seed(d + used)
    T, H, Hkv, page = 21, 4, 2, 32
    q, k, v, dq, dk = (torch.randn(T, n, d, generator=g).to(torch.bfloat16).cuda() for n in (H, Hkv, Hkv, H, Hkv))
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in "qk")
    rope = binding.Rope.of(d, 500000.0, axes=torch.arange(d // 2) % used)
    assert rope.axes == used
    all_of_them = torch.randint(0, 90000, (4, T), generator=g, dtype=torch.int32).cuda()
    got = []
    for pos in (all_of_them[:used].contiguous(), all_of_them):
        pool = binding.KvPages.empty(1, 4, Hkv, d, page, 1, 4, dtype)
        one = torch.tensor([0], dtype=torch.int32, device="cuda")
        pool.reserve(one, one + T)
        turned = pool.append(0, q, k, v, torch.tensor([0, T], dtype=torch.int32, device="cuda"), None, rope, wq, wk, positions=pos)
        got.append([turned, pool.k_pages.view(torch.uint8), pool.v_pages.view(torch.uint8), *binding.qk_norm_rotate(q, k, pos, rope, wq, wk),
                    *binding.qk_norm_rotate_backward(dq, dk, q, k, pos, rope, wq, wk)])
    assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.equal(got[0][0], got[0][3])
    for bad in (all_of_them[:, :20].contiguous(), all_of_them[:used - 1].contiguous(), all_of_them.repeat(3, 1), all_of_them[None]):
        with pytest.raises(ValueError):
            binding.qk_norm_rotate(q, k, bad, rope, wq, wk)
