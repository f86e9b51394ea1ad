"""Bounds that the sequences do not keep, and batches whose parts of keys share a small workspace."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2502_18394_amd import binding
from test_gpu_attend import DT, check, make, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("max_new,news", [(1, [1, 3, 1]), (2, [1, 5, 2]), (4, [4, 4, 40]), (40, [40, 300, 7]), (70, [1, 2, 500, 70])])
@pytest.mark.parametrize("most", [100, 5000])
def test_more_new_tokens_than_the_bound(io, max_new, news, most):
    """Rows of a sequence that has more are right or left as they are, whatever an earlier call left in the workspace."""
    print(f"case {io} max_new={max_new} {news} most={most}", flush=True)
    lens = [n + m for n, m in zip(news, (600, 900, 77, 300))]
    pool, rows = make(io, 64, 1, 16, lens, 3)
    q, start = queries(news, 4, 64, io, 5)
    other = torch.randn(q.shape, generator=torch.Generator().manual_seed(9)).to(q.dtype).cuda()
    for n in (max_new, max(news)):
        pool.attend(0, other, start, max_new=n, max_len=5000)
    out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 7.0, device="cuda")
    pool.attend(0, q, start, max_new=max_new, max_len=most, out=out, lse=lse)
    at = 0
    for b, n in enumerate(news):
        here = slice(at, at + n)
        at += n
        # a workgroup's rows end with a token's last head here, so a sequence's first tokens are done and the others left
        left = (lse[here] == 7.0).all(-1)
        done = n - int(left.sum())
        assert done == n if n <= max_new else done < n
        assert not left[:done].any() and left[done:].all() and (out[here][done:] == 9.0).all()
        k, v = (x[:lens[b] - n + done] for x in rows[b])
        check(out[here][:done], lse[here][:done], q[here][:done], [done], [(k, v)], 0.125, DT[io])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("news,lens", [([1, 2], [9000, 4100]), ([3, 3], [4096, 8200]), ([1, 90], [8193, 5000]), ([60, 50], [4500, 9001])])
@pytest.mark.parametrize("window", [0, 4500])
def test_lengths_above_their_bound(io, news, lens, window):
    """They cost time only: a workgroup then walks more page numbers than it holds at once."""
    print(f"case {io} {news} {lens} window={window}", flush=True)
    pool, rows = make(io, 64, 1, 16, lens, 4)
    q, start = queries(news, 2, 64, io, 6)
    pick = sorted({0, news[0] - 1, news[0], sum(news) - 1})
    for most in (1, 300):
        out, lse = pool.attend(0, q, start, max_new=max(news), max_len=most, window=window, want_lse=True)
        for t in pick:
            b = int(t >= news[0])
            p = lens[b] - news[b] + t - b * news[0]
            check(out[t:t + 1], lse[t:t + 1], q[t:t + 1], [1], [(rows[b][0][:p + 1], rows[b][1][:p + 1])], 0.125, DT[io], window)


@pytest.mark.parametrize("io,d,H,Hkv", [("bf16", 64, 32, 2), ("bf16", 128, 16, 4), ("f32", 64, 16, 8), ("bf16", 64, 32, 1)])
@pytest.mark.parametrize("news,lens", [([1, 700, 3, 0, 1500, 1, 200], [9100, 9500, 20, 500, 8000, 4000, 14000]), ([2000, 1, 2500, 2300], [9000, 70, 9700, 8800])])
def test_parts_share_a_workspace(io, d, H, Hkv, news, lens):
    """A bound of lengths far above most of them: rows have as many parts as their own sequence needs, and fewer where all parts together would not fit."""
    print(f"case {io} d={d} H={H} Hkv={Hkv} {news}", flush=True)
    most = 131072
    pool, rows = make(io, d, Hkv, 64, lens, d + H)
    q, start = queries(news, H, d, io, 7)
    T = sum(news)
    need = max(pool.attend_workspace_bytes(len(news), T, H, max(news), most, window) for window in (0, 6000))
    assert need <= max(128 << 20, 5 * T * H // 2 * (4 * d + 8)) + (256 << 20) + 8 * T * H + 4096
    given = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")       # NaN everywhere, counts of -1
    behind = torch.full((1 << 20,), 77, dtype=torch.uint8, device="cuda")
    for window in (0, 6000):
        out, lse = pool.attend(0, q, start, max_new=max(news), max_len=most, window=window, want_lse=True, ws=given)
        again = pool.attend(0, q, start, max_new=max(news), max_len=most, window=window, ws=given)
        assert torch.equal(out, again) and torch.isfinite(out).all() and torch.isfinite(lse).all()
        r = np.random.default_rng(3)
        for b, (n, m) in enumerate(zip(news, lens)):
            for i in sorted({0, n - 1, *r.integers(0, n, 3).tolist()}) if n else []:
                t, p = int(start[b]) + i, m - n + i
                check(out[t:t + 1], lse[t:t + 1], q[t:t + 1], [1], [(rows[b][0][:p + 1], rows[b][1][:p + 1])], d ** -0.5, DT[io], window)
    assert (behind == 77).all()


def test_bounds_so_loose_that_parts_are_left_out():
    """64 single tokens at the front of a batch that could be 65536 new tokens of sequences of 131072: as many parts as a launch can have."""
    H, Hkv, B = 32, 8, 64
    lens = [300 + 37 * b for b in range(B)]
    pool, rows = make("bf16", 64, Hkv, 64, lens, 2)
    q, start = queries([1] * B, H, 64, "bf16", 3)
    wide = torch.cat((q, q.new_zeros((1 << 16) - B, H, 64)))
    out = torch.full_like(wide, 9.0)
    _, lse = pool.attend(0, wide, start, max_new=1 << 16, max_len=131072, out=out, want_lse=True)
    assert (out[B:] == 9.0).all()
    check(out[:B], lse[:B], q, [1] * B, rows, 0.125, DT["bf16"])
