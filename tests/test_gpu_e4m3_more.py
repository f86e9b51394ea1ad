"""Pages of 8 bits on the GPU: what lies where nobody has written, scales among it, takes no part; tiles of 256 rows; appends of thousands of tokens."""
import numpy as np
import pytest
import torch

import e4m3_ref as ref
import paged_ref
from paper_2502_18394_amd import binding
from test_gpu_attend import FEW, MIXED, SINGLES, check, queries
from test_gpu_e4m3 import BF16, F8, NAN, _check_block, _ints, make
from test_gpu_heads import _turn_size

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


# ---------------------------------------------------------------- wide tiles
def _check_some(out, lse, q, start, news, lens, rows, d, window, there=None, skip=(), seed=5):
    """Rows at the ends and picked at random; of the sequences in `skip` not the last two."""
    pick = np.random.default_rng(seed)
    for b, (n, m) in enumerate(zip(news, lens)):
        last = n - 2 if b in skip else n
        for i in sorted({0, n // 2, last - 1, *pick.integers(0, max(last, 1), 6)}) if n else []:
            at, p = int(start[b]) + int(i), m - n + int(i)
            alive = [there[b][:p + 1]] if there and b in there else None
            check(out[at:at + 1], lse[at:at + 1], q[at:at + 1], [1], [(rows[b][0][:p + 1], rows[b][1][:p + 1])], d ** -0.5, BF16, window, alive)


@pytest.mark.parametrize("d,page", [(64, 64), (64, 16), (128, 16), (128, 64)])
@pytest.mark.parametrize("window", [0, 333])
def test_many_rows_of_many_heads(d, page, window):
    """A mixed batch with work for every compute unit, which has tiles of 256 rows: an absent page, a NaN value where most rows do not see it."""
    print(f"case d={d} page={page} window={window}", flush=True)
    news, lens, H, Hkv = [700, 1, 513, 0, 640, 600, 700, 255], [900, 77, 513, 40, 1000, 601, 700, 300], 32, 16
    pool, rows = make(d, Hkv, page, lens, page + d)
    at = lens[4] - 2                                         # the last token but one
    pool.v_pages.view(torch.uint8)[0, int(pool.table[4, at // page]), :, at % page // 16, 7, at % 16] = NAN
    pool.table[6, 2] = -1
    there = np.ones(700, bool)
    there[2 * page:3 * page] = False
    q, start = queries(news, H, d, "bf16", 3)
    out, lse = pool.attend(0, q, start, max_new=700, max_len=1000, window=window, want_lse=True)
    _check_some(out, lse, q, start, news, lens, rows, d, window, {6: there}, (4,))
    end = int(start[5])
    assert out[end - 2:end, :, 7].isnan().all()
    out[end - 2:end, :, 7] = 0
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [0, 8200])
def test_a_chunk_of_many_rows_over_a_long_cache(d, window):
    """One sequence whose tiles of 256 rows have their keys divided; keys beyond a whole tile."""
    print(f"case d={d} window={window}", flush=True)
    n, m, H, Hkv = 1024, 9241, 32, 16
    pool, rows = make(d, Hkv, 32, [m], d)
    there = np.ones(m, bool)
    for j, value in ((0, -1), (100, pool.pages), (280, -3)):
        pool.table[0, j] = value
        there[32 * j:32 * j + 32] = False
    q, start = queries([n], H, d, "bf16", 4)
    out, lse = pool.attend(0, q, start, max_new=n, max_len=m, window=window, want_lse=True)
    _check_some(out, lse, q, start, [n], [m], rows, d, window, {0: there})
    assert torch.isfinite(out).all()


# ---------------------------------------------------------------- long appends
@pytest.mark.parametrize("d,Hkv", [(64, 9), (64, 2), (128, 5)])
@pytest.mark.parametrize("T", [3900, 6100, 9001, 11000])
def test_append_of_many_tokens(d, Hkv, T):
    """Prompts whose blocks' heads have four workgroups, two, one, and one together with the queries: key heads in several passes of a workgroup, one of them with
    half the heads.  The first sequence begins inside a block whose scale grows."""
    print(f"case d={d} Hkv={Hkv} T={T}", flush=True)
    H, page, had, news = 2 * Hkv, 64, [5, 0, 30], [T - 1200, 1, 1199]
    g = torch.Generator().manual_seed(T + d + Hkv)
    pool = binding.KvPages.empty(1, T // page + 6, Hkv, d, page, 3, T // page + 2, F8)
    pool.reserve(_ints([0, 1, 2]), _ints(had))
    pool.append(0, *(torch.zeros(sum(had), n, d, dtype=BF16, device="cuda") for n in (H, Hkv, Hkv)), _ints([0, 5, 5, 35]))
    pool.reserve(_ints([0, 1, 2]), _ints(news))
    q, k, v = (torch.randn(T, n, d, generator=g).mul(torch.exp2(2 * torch.randn(T, 1, 1, generator=g))).to(BF16).cuda() for n in (H, Hkv, Hkv))
    w = [(1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in "qk"]
    rope = binding.Rope.of(d, 500000.0)
    out = pool.append(0, q, k, v, torch.tensor([0] + news).cumsum(0).int().cuda(), None, rope, *w)
    pos = torch.cat([torch.arange(a, a + n) for a, n in zip(had, news)]).int()
    assert int(pool.status[0]) == 0 and torch.equal(out, binding.qk_norm_rotate(q, k, pos.cuda(), rope, *w)[0])
    at, pick = 0, np.random.default_rng(T)
    for s, (a, n) in enumerate(zip(had, news)):
        whole = Rows(pool, s, a + n)
        last = (a + n - 1) // 16
        for block in sorted({0, 1, last - 1, last, *pick.integers(0, last + 1, 4)}):
            if not 0 <= block <= last:
                continue
            lo, hi = max(16 * block, a), min(16 * block + 16, a + n)
            if hi <= lo:
                continue
            new = slice(at + lo - a, at + hi - a)
            x, p = k[new].double().cpu().numpy(), pos[new].numpy()
            plain = paged_ref.heads(x, paged_ref.f64(w[1]), p, np.zeros(0), 1e-6)
            k64, size = paged_ref.heads(x, paged_ref.f64(w[1]), p, paged_ref.f64(rope.inv_freq), 1e-6), _turn_size(plain, d // 2, False)
            zeros = np.zeros((lo - 16 * block, Hkv, d))
            k64, size, v64 = (np.concatenate((zeros, y)) for y in (k64, size, v[new].double().cpu().numpy()))
            _check_block(whole.at(block), 0, 0, 0, hi - 16 * block, [lo - 16 * block] if lo > 16 * block else [], k64, size, v64, d)
        at += n


class Rows:
    """One sequence's pages on the host; at(block): the 16 tokens of one block as a pool of one page."""

    def __init__(self, pool, row, n):
        self.pool, numbers = pool, pool.table[row, :-(-n // pool.page)].long()
        self.k, self.v, self.scales = pool.k_pages.view(torch.uint8)[:, numbers].cpu(), pool.v_pages.view(torch.uint8)[:, numbers].cpu(), pool.scales[:, numbers].cpu()

    def at(self, block):
        one = Rows.__new__(Rows)
        p, i = block * 16 // self.pool.page, block % (self.pool.page // 16)
        one.page, one.Hkv, one.d = 16, self.pool.Hkv, self.pool.d
        one.table = torch.zeros(1, 1, dtype=torch.int32)
        one.k_pages = self.k[:, p:p + 1, :, :, 16 * i:16 * i + 16].contiguous().view(F8)
        one.v_pages = self.v[:, p:p + 1, :, i:i + 1].contiguous().view(F8)
        one.scales = self.scales[:, p:p + 1, :, i:i + 1].contiguous()
        return one
