"""Bounds that the sequences do not keep."""
import pytest
import torch

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
