"""Pages of a pool on the GPU against the plain bookkeeping: every word of it, and every byte of the pages."""
import random

import pytest
import torch

import paged_ref as ref
from paper_2502_18394_amd import binding

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Both:
    """A pool and its plain double; check() compares all of both."""

    def __init__(self, io="bf16", layers=2, pages=40, Hkv=2, d=64, page=16, seqs=8, max_pages=9, seed=0):
        self.pool = binding.KvPages.empty(layers, pages, Hkv, d, page, seqs, max_pages, DT[io])
        g = torch.Generator(device="cuda").manual_seed(seed)
        for x in (self.pool.k_pages, self.pool.v_pages):
            x.normal_(generator=g)
        self.k, self.v = self.pool.k_pages.cpu().clone(), self.pool.v_pages.cpu().clone()
        self.book, self.E = ref.Book(seqs, pages, max_pages, page), ref.per_group(DT[io])

    def copy(self, moves):
        for a, b in moves:
            self.k[:, b], self.v[:, b] = self.k[:, a], self.v[:, a]

    def reserve(self, seqs, add):
        self.pool.reserve(_ints(seqs), _ints(add))
        self.book.reserve(seqs, add)

    def fork(self, src, dst):
        self.pool.fork(_ints(src), _ints(dst))
        for a, b, rest in self.book.fork(src, dst):
            some = -(-rest // self.E) * self.E
            self.k[:, b, :, :, :some] = self.k[:, a, :, :, :some]
            self.v[:, b, :, :some // self.E] = self.v[:, a, :, :some // self.E]

    def free(self, seqs):
        self.pool.free(_ints(seqs))
        self.book.free(seqs)

    def compact(self):
        self.pool.compact()
        self.copy(self.book.compact())

    def check(self):
        assert self.pool.book.tolist() == self.book.words()
        assert torch.equal(self.pool.k_pages.cpu(), self.k) and torch.equal(self.pool.v_pages.cpu(), self.v)


@pytest.mark.parametrize("io,d,page,Hkv", [("bf16", 64, 16, 2), ("f32", 64, 16, 1), ("bf16", 128, 64, 3), ("f32", 128, 32, 2), ("bf16", 64, 256, 1)])
def test_a_life_of_sequences(io, d, page, Hkv):
    print(f"case {io} d={d} page={page}", flush=True)
    b = Both(io, layers=2, pages=37, Hkv=Hkv, d=d, page=page, seqs=9, max_pages=8)
    b.check()
    b.reserve([4, 0, 7], [page * 3 + 5, 1, 0])
    b.check()
    b.reserve([0, 4], [page - 1, page - 5])                 # up to full pages, exactly
    b.check()
    b.reserve([0], [1])
    b.fork([4, 0, 0, 7], [1, 2, 8, 3])                       # a full one, two of one parent, one of nothing
    b.check()
    b.reserve([2, 8], [page, 3])
    b.free([4, 5])                                          # its pages live on in the child; an empty one
    b.check()
    b.free([0, 0, 0])                                       # once, however often it is listed
    b.check()
    b.compact()
    b.check()
    b.compact()                                             # nothing left to move
    b.check()
    b.fork([2], [0])
    b.free([1, 2, 8, 0])
    b.check()
    b.compact()
    b.check()


def test_a_random_life():
    r = random.Random(7)
    b = Both(layers=1, pages=60, seqs=20, max_pages=6, Hkv=1)
    for step in range(60):
        what = r.choice(["reserve", "reserve", "fork", "free", "compact"])
        print(f"step {step} {what}", flush=True)
        live, empty = [s for s in range(20) if b.book.lens[s]], [s for s in range(20) if not b.book.lens[s]]
        if what == "reserve":
            s = r.sample(range(20), r.randint(1, 6))
            b.reserve(s, [r.randint(0, 30) for _ in s])
        elif what == "fork" and live and empty:
            dst = r.sample(empty, r.randint(1, min(4, len(empty))))
            b.fork([r.choice(live) for _ in dst], dst)
        elif what == "free" and live:
            b.free(r.sample(live, r.randint(1, min(3, len(live)))))
        else:
            b.compact()
        b.check()


def test_what_cannot_be_done_changes_nothing_but_the_status():
    b = Both(pages=6, max_pages=4)
    b.reserve([0, 1], [33, 17])                              # five of six pages
    b.check()
    b.reserve([0, 1, 2], [1, 20, 1])                         # needs two
    assert b.book.status[0] == 1
    b.check()
    b.reserve([0], [40])                                     # longer than a row
    assert b.book.status[0] == 3
    b.check()
    for seqs, add in (([0, 0], [1, 1]), ([8], [1]), ([-1], [1]), ([2], [-1])):
        b.reserve(seqs, add)
        b.check()
    assert b.book.status[0] == 7
    b.fork([0], [1])                                         # not empty
    assert b.book.status[0] == 15
    b.check()
    b.fork([0, 1], [2, 3])                                   # two last pages, one free
    b.fork([0, 2], [2, 3])                                   # read and written
    b.fork([0, 1], [2, 2])
    b.fork([9], [2])
    b.free([77, -3])
    b.check()
    b.pool.status.zero_()
    b.book.status = [0] * 8
    b.fork([0], [2])
    b.check()
    assert b.book.status[0] == 0


def test_copies_of_pages():
    b = Both("f32", layers=3, pages=50, Hkv=3, d=128, page=32)
    order = torch.randperm(50).tolist()
    src, dst = order[:20], order[20:40]
    b.pool.copy(_ints(src), _ints(dst))
    b.copy(zip(src, dst))
    b.check()
    b.pool.copy(_ints([3, 50, -1, 4]), _ints([50, 2, 1, 6]))  # out of range: left out
    b.copy([(4, 6)])
    b.book.status[0] = 4
    b.check()
    b.pool.copy(_ints([]), _ints([]))
    b.check()


def test_many_pages_and_sequences():
    """More pages and sequences than a workgroup looks at in one step."""
    b = Both(layers=1, pages=9001, Hkv=1, seqs=2100, max_pages=5, page=16)
    r = random.Random(1)
    for step in range(3):
        seqs = r.sample(range(2100), 1300)
        b.reserve(seqs, [r.randint(0, 20) for _ in seqs])
        b.check()
        b.free(r.sample(range(2100), 1100))
        b.check()
        live, empty = [s for s in range(2100) if b.book.lens[s]], [s for s in range(2100) if not b.book.lens[s]]
        b.fork([r.choice(live) for _ in range(1030)], empty[:1030])
        b.check()
        b.compact()
        b.check()


def test_page_calls_in_a_graph():
    """A captured tick (free, compact, reserve) replayed on other bookkeeping does what the calls do."""
    b = Both(pages=30, seqs=6, max_pages=5)
    b.reserve([0, 1, 2, 3], [20, 50, 70, 16])
    b.check()
    seqs, gone, add = _ints([0, 4]), _ints([1]), _ints([3, 30])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kept = b.pool.book.clone(), b.pool.k_pages.clone(), b.pool.v_pages.clone()
    with torch.cuda.stream(side):                            # workspaces exist before the capture
        b.pool.compact()
        for x, y in zip((b.pool.book, b.pool.k_pages, b.pool.v_pages), kept):
            x.copy_(y)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.pool.free(gone)
        b.pool.compact()
        b.pool.reserve(seqs, add)
    torch.cuda.synchronize()
    b.check()                                                # nothing ran yet
    for s, g, a in (([0, 4], [1], [3, 30]), ([1, 5], [2], [40, 0]), ([0, 3], [4], [1, 1])):
        seqs.copy_(_ints(s)), gone.copy_(_ints(g)), add.copy_(_ints(a))
        graph.replay()
        b.book.free(g)
        b.copy(b.book.compact())
        b.book.reserve(s, a)
        b.check()

