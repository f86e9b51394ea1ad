"""What must not happen to tokens that are there."""
import pytest
import torch

from paper_2502_18394_amd import binding

pytestmark = pytest.mark.gpu
H, Hkv, d, page = 4, 2, 64, 16


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pool(pages, seqs, max_pages, io=torch.bfloat16, layers=2):
    pool = binding.KvPages.empty(layers, pages, Hkv, d, page, seqs, max_pages, io)
    g = torch.Generator(device="cuda").manual_seed(pages)
    for x in (pool.k_pages, pool.v_pages):
        x.normal_(generator=g)
    return pool


def _tokens(T, io=torch.bfloat16, seed=1):
    row = torch.randn(T, H + 2 * Hkv, d, generator=torch.Generator().manual_seed(seed)).to(io).cuda()
    return row[:, :H], row[:, H:H + Hkv], row[:, H + Hkv:]


def _all(pool):
    return [x.clone() for x in (pool.k_pages, pool.v_pages, pool.book)]


def _untouched(pool, before, status):
    now = _all(pool)
    assert torch.equal(now[0], before[0]) and torch.equal(now[1], before[1])
    assert torch.equal(now[2][1:], before[2][1:]) and int(now[2][0]) == status


@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("why,status", [("pages", 1), ("length", 2), ("argument", 4)])
def test_a_step_whose_reserve_failed_writes_nothing(io, why, status):
    print(f"case {why} {io}", flush=True)
    pool = _pool(6 if why == "pages" else 40, 4, 3, io)
    pool.reserve(_ints(0, 1, 2), _ints(32, 31, 48 if why == "length" else 20))
    before = _all(pool)
    assert int(pool.status[0]) == 0
    seqs = _ints(0, 1, 2) if why != "argument" else _ints(0, 1, 0)
    pool.reserve(seqs, _ints(1, 1, 1))                       # the second has room in its last page; the call as a whole cannot be done
    _untouched(pool, before, status)
    rope, start = binding.Rope.of(d), _ints(0, 1, 2, 3)
    for layer in range(2):
        pool.append(layer, *_tokens(3, io), start, _ints(0, 1, 2), rope)
    _untouched(pool, before, status)
    # the caller has seen it: what has room goes on
    pool.status.zero_()
    pool.reserve(_ints(1), _ints(1))
    pool.append(1, *_tokens(1, io), start[:2], _ints(1), rope)
    assert int(pool.lens[1]) == 32 and int(pool.status[0]) == 0
    number, at = int(pool.table[1, 1]), 15
    assert not torch.equal(pool.k_pages[1, number, :, :, at], before[0][1, number, :, :, at])
    pool.k_pages[1, number, :, :, at] = before[0][1, number, :, :, at]
    E = 8 if io == torch.bfloat16 else 4
    pool.v_pages[1, number, :, at // E, :, at % E] = before[1][1, number, :, at // E, :, at % E]
    assert torch.equal(pool.k_pages, before[0]) and torch.equal(pool.v_pages, before[1])


def test_a_captured_step_that_runs_out_of_pages():
    """A full prompt forked into samples whose captured steps take the last pages: from then on every replay leaves all bytes as they are."""
    pool = _pool(5, 3, 4)
    pool.reserve(_ints(0), _ints(2 * page))
    pool.fork(_ints(0, 0), _ints(1, 2))                      # both pages shared by three
    row = torch.randn(2, H + 2 * Hkv, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q, k, v = row.split((H, Hkv, Hkv), 1)
    seqs, one, start, rope = _ints(1, 2), _ints(1, 1), _ints(0, 1, 2), binding.Rope.of(d)

    def step():
        pool.reserve(seqs, one)
        pool.append(0, q, k, v, start, seqs, rope)

    before = _all(pool)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        for x, y in zip((pool.k_pages, pool.v_pages, pool.book), before):
            x.copy_(y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(page):
        row.normal_()
        graph.replay()
    assert pool.lens.tolist() == [2 * page, 3 * page, 3 * page] and int(pool.status[0]) == 0
    full = _all(pool)
    for _ in range(3):
        row.normal_()
        graph.replay()
        torch.cuda.synchronize()
        _untouched(pool, full, binding.KvPages.NO_PAGES)


def test_pages_with_several_users_are_not_written():
    pool = _pool(8, 3, 4)
    pool.reserve(_ints(0), _ints(2 * page))
    pool.fork(_ints(0), _ints(1))
    before = _all(pool)
    start, rope = _ints(0, 3), binding.Rope.of(d)
    for s in (0, 1):                                         # no reserve: the last tokens of both lie in a page of both
        pool.append(1, *_tokens(3), start, _ints(s), rope)
        _untouched(pool, before, binding.KvPages.SHARED)
    pool.status.zero_()
    pool.reserve(_ints(1), _ints(3))
    pool.append(1, *_tokens(3), start, _ints(1), rope)
    assert int(pool.status[0]) == 0
    number = int(pool.table[1, 2])
    assert not torch.equal(pool.k_pages[1, number, :, :, :3], before[0][1, number, :, :, :3])
    rest = torch.ones(8, dtype=torch.bool)
    rest[number] = False
    assert torch.equal(pool.k_pages[:, rest], before[0][:, rest]) and torch.equal(pool.v_pages[:, rest], before[1][:, rest])


@pytest.mark.parametrize("absent", [-1, 8, 2 ** 31 - 1])
def test_a_fork_of_a_last_page_that_is_absent(absent):
    """The child is what its parent is: the tokens of a page outside the pool are absent in both, and no page is taken for them."""
    pool = _pool(8, 4, 3)
    pool.reserve(_ints(0, 1), _ints(page + 5, 7))
    pool.table[0, 1] = absent
    refs = pool.refs.clone()
    before = _all(pool)
    pool.fork(_ints(0, 1), _ints(2, 3))
    assert pool.table[2].tolist() == [int(before[2][12 + 8]), absent, -1] and pool.lens.tolist() == [page + 5, 7, page + 5, 7]
    fresh = int(pool.table[3, 0])
    refs[int(pool.table[0, 0])] += 1
    refs[fresh] += 1
    assert torch.equal(pool.refs, refs) and pool.status[:2].tolist() == [0, 1]
    q = torch.randn(1, H, d, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    one = _ints(0, 1)
    assert torch.equal(pool.attend(0, q, one, _ints(0), 1), pool.attend(0, q, one, _ints(2), 1))
    pool.free(_ints(0, 1, 2, 3))
    assert int((pool.refs > 0).sum()) == 1                    # the page that the table lost
