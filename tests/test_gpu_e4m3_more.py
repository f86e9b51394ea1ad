"""Pages of 8 bits on the GPU: what lies where nobody has written, scales among it, takes no part."""
import numpy as np
import pytest
import torch

import e4m3_ref as ref
from paper_2502_18394_amd import binding
from test_gpu_attend import FEW, MIXED, SINGLES, check, queries
from test_gpu_e4m3 import BF16, F8, _ints, make

pytestmark = pytest.mark.gpu


def _unwritten(pool, lens):
    """Scales of blocks that no token has reached: NaN, infinities, all bits set, zero."""
    live = torch.zeros(pool.pages, pool.page // 16, dtype=torch.bool)
    table = pool.table.cpu()
    for s, n in enumerate(lens):
        for first in range(0, n, 16):
            live[int(table[s, first // pool.page]), first % pool.page // 16] = True
    bits = torch.tensor([0x7fc00000, 0x7f800000, -0x800000, -1, 0], dtype=torch.int32)
    bits = bits[torch.arange(pool.scales.numel()) % len(bits)].view(torch.float32).view(pool.scales.shape).cuda()
    gone = ~live.cuda()[None, :, None, :, None]
    pool.scales.copy_(torch.where(gone, bits, pool.scales))
    assert torch.isnan(pool.scales).any()


@pytest.mark.parametrize("d,page", [(64, 32), (64, 256), (128, 64), (128, 256)])
@pytest.mark.parametrize("name", ["SINGLES", "FEW", "MIXED"])
def test_scales_of_blocks_without_tokens(d, page, name):
    print(f"case {name} d={d} page={page}", flush=True)
    news, lens = {"SINGLES": SINGLES, "FEW": FEW, "MIXED": MIXED}[name]
    pool, rows = make(d, 2, page, lens, d + page)
    _unwritten(pool, lens)
    q, start = queries(news, 4, d, "bf16", page)
    for window in (0, 50):
        out, lse = pool.attend(0, q, start, max_new=max(news), max_len=max(lens), window=window, want_lse=True)
        check(out, lse, q, news, rows, d ** -0.5, BF16, window)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [4, 8, 12, 16, 17, 40])
def test_scales_of_blocks_without_tokens_some_rows(d, n):
    """Four rows a token: groups of 16 that share keys and values, and tiles; sequences that end in every block of a page."""
    print(f"case d={d} n={n}", flush=True)
    lens = [700, 641, n, 64 + n, 1000 + n, 17]
    news = [n, 1, n, n, n, min(n, 17)]
    pool, rows = make(d, 1, 128, lens, d + n)
    _unwritten(pool, lens)
    q, start = queries(news, 4, d, "bf16", n)
    out, lse = pool.attend(0, q, start, max_new=n, max_len=max(lens), want_lse=True)
    check(out, lse, q, news, rows, d ** -0.5, BF16)


@pytest.mark.parametrize("n", [1, 9, 40])
def test_a_pool_of_memory_that_nobody_has_cleared(n):
    """Arrays as an allocator gives them, at worst: all bits set.  What append writes is all that attention sees."""
    layers, pages, Hkv, d, page, m = 1, 12, 2, 64, 64, 150
    k, v = (torch.full(shape, 255, dtype=torch.uint8, device="cuda").view(F8) for shape in ((layers, pages, Hkv, d // 16, page, 16), (layers, pages, Hkv, page // 16, d, 16)))
    scales = torch.full((layers, pages, Hkv, page // 16, 2), -1, dtype=torch.int32, device="cuda").view(torch.float32)
    pool = binding.KvPages(k, v, torch.empty(8 + 2 + pages + 2 * 6, dtype=torch.int32, device="cuda"), 2, 6, scales)
    pool.reset()
    g = torch.Generator().manual_seed(n)
    rows = [torch.randn(2 * m, heads, d, generator=g).to(BF16).cuda() for heads in (4, Hkv, Hkv)]
    pool.reserve(_ints([0, 1]), _ints([m, m]))
    pool.append(0, *rows, _ints([0, m, 2 * m]))
    kv = [ref.rows(pool, 0, s, m)[:2] for s in (0, 1)]
    assert all(np.isfinite(x).all() for pair in kv for x in pair)
    q, start = queries([n, n], 4, d, "bf16", n)
    out, lse = pool.attend(0, q, start, max_new=n, max_len=m, want_lse=True)
    check(out, lse, q, [n, n], kv, 0.125, BF16)
