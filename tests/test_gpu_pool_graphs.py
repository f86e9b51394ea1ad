"""Captured calls on a pool whose eager calls come to need a larger workspace."""
import pytest
import torch

from paper_2502_18394_amd import binding
from test_gpu_attend import make, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("warm", [True, False])
def test_a_graph_keeps_its_workspace(warm):
    """A decode step of split keys is captured; an eager chunk on the same pool needs more; memory that the pool gave back belongs to others from
    then on, and replays write none of it."""
    H, d, lens = 4, 64, [3000, 9000]
    pool, _ = make("bf16", d, 1, 64, lens, 1)
    q, start = queries([1, 1], H, d, "bf16", 2)
    chunk, wide = queries([40, 300], H, d, "bf16", 3)
    step = lambda: pool.attend(0, q, start, max_new=1, max_len=9000, want_lse=True)
    want, want_lse = binding.KvPages(pool.k_pages, pool.v_pages, pool.book, 2, pool.max_pages).attend(0, q, start, max_new=1, max_len=9000, want_lse=True)
    if warm:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step()
    small = pool.attend_workspace_bytes(2, 2, H, 1, 9000)
    assert pool.attend_workspace_bytes(2, 340, H, 300, 9000) > small + 512
    first = pool.attend(0, chunk, wide, max_new=300, max_len=9000)
    torch.cuda.synchronize()
    taken = [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for n in 8 * [small + 256, small, small + 512, 1 << 20]]
    for _ in range(4):
        out.zero_(), lse.zero_()
        graph.replay()
        assert torch.equal(pool.attend(0, chunk, wide, max_new=300, max_len=9000), first)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert all(bool((x == 77).all()) for x in taken)
    del graph, out, lse                                      # the pool goes on without it
    assert torch.equal(pool.attend(0, chunk, wide, max_new=300, max_len=9000), first)
    assert torch.equal(step()[0], want)


def test_page_calls_in_a_graph_keep_their_workspace():
    """Captured reserves beside eager calls with longer lists."""
    def filled():
        pool = binding.KvPages.empty(1, 30, 1, 64, 16, 200, 8)
        pool.reserve(torch.arange(3, dtype=torch.int32, device="cuda"), torch.tensor([20, 5, 16], dtype=torch.int32, device="cuda"))
        return pool

    one, two = filled(), filled()
    seqs, add = torch.tensor([0, 2], dtype=torch.int32, device="cuda"), torch.tensor([3, 9], dtype=torch.int32, device="cuda")
    many, none = torch.arange(200, dtype=torch.int32, device="cuda"), torch.zeros(200, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.reserve(seqs, add)
    for _ in range(4):
        one.reserve(many, none)                              # asks for more than the captured call did
        taken = [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for n in 16 * [512, 1024, 2048]]
        graph.replay()
        two.reserve(seqs, add)
        torch.cuda.synchronize()
        assert torch.equal(one.book, two.book) and all(bool((x == 77).all()) for x in taken)


def test_a_capture_on_a_stream_that_is_given():
    """The calls' own `stream` is the one being captured."""
    H, d, lens = 4, 64, [9000]
    pool, _ = make("bf16", d, 1, 64, lens, 1)
    q, start = queries([1], H, d, "bf16", 2)
    chunk, wide = queries([500], H, d, "bf16", 3)
    want = pool.attend(0, q, start, max_new=1, max_len=9000)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = pool.attend(0, q, start, max_new=1, max_len=9000, stream=side)
    first = pool.attend(0, chunk, wide, max_new=500, max_len=9000)
    small = pool.attend_workspace_bytes(1, 1, H, 1, 9000)
    taken = [torch.full((small + 256,), 77, dtype=torch.uint8, device="cuda") for _ in range(8)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(pool.attend(0, chunk, wide, max_new=500, max_len=9000), first)
    assert all(bool((x == 77).all()) for x in taken)
