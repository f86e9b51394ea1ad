"""Attention of new tokens over pages on the GPU against the 64-bit form."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2502_18394_amd import binding

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U32 = 2.0 ** -24


def make(io, d, Hkv, page, lens, seed, fill=float("nan"), layers=1, scale=1.0):
    """A pool whose sequences hold keys and values of normal distribution, everything else `fill`; with the keys and values, [m, Hkv, d] each."""
    g = torch.Generator().manual_seed(seed)
    M, P = max(1, max(-(-n // page) for n in lens)) + 1, sum(-(-n // page) for n in lens) + 4
    pool = binding.KvPages.empty(layers, P, Hkv, d, page, len(lens), M, DT[io])
    E = ref.per_group(DT[io])
    k, v = torch.full((P, page, Hkv, d), fill), torch.full((P, page, Hkv, d), fill)
    order = torch.randperm(P, generator=g)
    table, refs, rows, at = pool.table.cpu(), pool.refs.cpu(), [], 0
    for s, n in enumerate(lens):
        m = -(-n // page)
        mine = order[at:at + m]
        at += m
        table[s, :m], refs[mine] = mine.int(), 1
        a, b = (torch.randn(n, Hkv, d, generator=g) * x for x in (scale, 1.0))
        for x, y in ((k, a), (v, b)):
            whole = x[mine].reshape(m * page, Hkv, d)
            whole[:n] = y.to(DT[io]).float()
            x[mine] = whole.reshape(m, page, Hkv, d)
        rows.append((ref.f64(a.to(DT[io])), ref.f64(b.to(DT[io]))))
    layer = layers - 1
    pool.k_pages.fill_(fill)
    pool.v_pages.fill_(fill)
    pool.k_pages[layer] = k.view(P, page, Hkv, d // E, E).permute(0, 2, 3, 1, 4).to(DT[io]).cuda()
    pool.v_pages[layer] = v.view(P, page // E, E, Hkv, d).permute(0, 3, 1, 4, 2).to(DT[io]).cuda()
    pool.table.copy_(table)
    pool.refs.copy_(refs)
    pool.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return pool, rows


def queries(news, H, d, io, seed, scale=1.5):
    g = torch.Generator().manual_seed(seed + 1)
    start = torch.tensor([0] + list(news)).cumsum(0).int()
    q = (torch.randn(int(start[-1]), H, d, generator=g) * scale).to(DT[io]).cuda()
    return q, start.cuda()


def check(out, lse, q, news, rows, scale, dtype, window=0, there=None, seqs=None):
    at = 0
    for b, n in enumerate(news):
        k, v = rows[seqs[b] if seqs else b]
        if n:
            x = ref.f64(q[at:at + n])
            alive = None if there is None else there[b]
            want, want_lse = ref.attend(x, k, v, scale, window, alive)
            tol = ref.attend_bound(x, k, v, scale, dtype, window, alive)
            got = ref.f64(out[at:at + n])
            assert np.isfinite(got).all(), f"sequence {b}: not finite"
            assert (np.abs(got - want) <= tol).all(), f"sequence {b}: {float((np.abs(got - want) / np.maximum(tol, 1e-30)).max())} of the bound"
            if lse is not None:
                got = ref.f64(lse[at:at + n])
                none = np.isneginf(want_lse)
                assert (np.isneginf(got) == none).all()
                most = np.abs(x).max() * max(np.abs(k).max(), 1e-30) * scale * (x.shape[2] + 4) * U32 * x.shape[2] if len(k) else 0.0
                assert (np.abs(got[~none] - want_lse[~none]) <= most + (len(k) + 16) * U32 + 4 * U32 * np.abs(want_lse[~none])).all()
        at += n


# new tokens and tokens of each sequence: single tokens at every border of a page, a step and a tile; nothing; more new tokens than there are tokens
SINGLES = ([1] * 14, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300])
FEW = ([3, 1, 0, 5, 8, 2], [3, 40, 17, 300, 8, 1])
MANY = ([70, 33, 129, 64], [70, 200, 129, 65])
MIXED = ([1, 150, 0, 2, 40], [700, 150, 30, 2, 333])
SHORT = ([5, 40, 2], [3, 7, 0])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 16), (64, 64), (128, 32), (128, 128)])
@pytest.mark.parametrize("H,Hkv", [(4, 1), (2, 2), (7, 1)])
@pytest.mark.parametrize("name", ["SINGLES", "FEW", "MANY", "MIXED", "SHORT"])
def test_against_the_definition(io, d, page, H, Hkv, name):
    print(f"case {name} {io} d={d} page={page} H={H} Hkv={Hkv}", flush=True)
    news, lens = globals()[name]
    pool, rows = make(io, d, Hkv, page, lens, d + page + H)
    q, start = queries(news, H, d, io, H)
    out, lse = pool.attend(0, q, start, max_new=max(news), max_len=max(lens), want_lse=True)
    check(out, lse, q, news, rows, d ** -0.5, DT[io])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 7, 64, 100])
@pytest.mark.parametrize("name", ["SINGLES", "FEW", "MANY", "MIXED"])
def test_windows(io, window, name):
    print(f"case {name} {io} window={window}", flush=True)
    news, lens = globals()[name]
    pool, rows = make(io, 64, 2, 16, lens, window)
    q, start = queries(news, 4, 64, io, window)
    out, lse = pool.attend(0, q, start, max_new=max(news), max_len=max(lens), window=window, want_lse=True)
    check(out, lse, q, news, rows, 0.125, DT[io], window)


@pytest.mark.parametrize("io,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("n", [1, 4, 9, 17, 60])
def test_keys_split_over_workgroups(io, d, n):
    """One sequence of many keys: its keys are divided, and the parts joined."""
    print(f"case {io} d={d} n={n}", flush=True)
    pool, rows = make(io, d, 1, 64, [2500], n + d, scale=2.0)
    q, start = queries([n], 2, d, io, n)
    assert pool.attend_workspace_bytes(1, n, 2, n, 2500) > 256
    for window in (0, 1111):
        out, lse = pool.attend(0, q, start, max_new=n, max_len=2500, window=window, want_lse=True)
        check(out, lse, q, [n], rows, d ** -0.5, DT[io], window)


@pytest.mark.parametrize("io,d,page", [("bf16", 64, 64), ("bf16", 128, 16), ("f32", 64, 32), ("f32", 128, 128), ("bf16", 64, 16)])
@pytest.mark.parametrize("window", [0, 333])
def test_many_rows_of_many_heads(io, d, page, window):
    """Batches with work for every compute unit, which have wider tiles: queries picked at random and at the ends, absent pages, NaN and infinities where rows
    do not see them."""
    print(f"case {io} d={d} page={page} window={window}", flush=True)
    news, lens, H, Hkv = [700, 1, 513, 0, 640, 600, 700, 255], [900, 77, 513, 40, 1000, 601, 700, 300], 32, 16
    pool, rows = make(io, d, Hkv, page, lens, page + d)
    for value in (float("nan"), float("inf")):                 # the last token but one of two sequences
        s = 4 if value == value else 0
        at = lens[s] - 2
        number, slot, E = int(pool.table[s, at // page]), at % page, ref.per_group(DT[io])
        pool.v_pages[0, number, :, slot // E, 7, slot % E] = value
    pool.table[6, 2] = -1
    there = np.ones(700, bool)
    there[2 * page:3 * page] = False
    q, start = queries(news, H, d, io, 3)
    out, lse = pool.attend(0, q, start, max_new=700, max_len=1000, window=window, want_lse=True)
    pick = np.random.default_rng(5)
    for b, (n, m) in enumerate(zip(news, lens)):
        last = n - 2 if b in (0, 4) else n                      # the last two rows of these see what is not finite
        for i in sorted({0, n // 2, last - 1, *pick.integers(0, max(last, 1), 6)}) if n else []:
            at, p = int(start[b]) + int(i), m - n + int(i)
            alive = [there[:p + 1]] if b == 6 else None
            check(out[at:at + 1], lse[at:at + 1], q[at:at + 1], [1], [(rows[b][0][:p + 1], rows[b][1][:p + 1])], d ** -0.5, DT[io], window, alive)
        if b in (0, 4):
            seen = out[int(start[b]) + n - 2:int(start[b]) + n, :, 7].float()
            assert not torch.isfinite(seen).any()
            assert torch.isfinite(out[int(start[b]):int(start[b]) + n - 2]).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 6, 50])
def test_bounds_that_are_wide_or_missing(io, n):
    """Bounds beyond the lengths change no value beyond the order of sums; other layers and rows of the table are not touched."""
    lens = [200, 77, 130]
    pool, rows = make(io, 64, 2, 32, lens, 5, layers=3)
    seqs = [2, 0]
    q, start = queries([n, n], 6, 64, io, 9)
    for args in (dict(max_new=n, max_len=200), dict(max_new=n, max_len=100000), dict()):
        out = pool.attend(2, q, start, torch.tensor(seqs, dtype=torch.int32, device="cuda"), **args)
        check(out, None, q, [n, n], rows, 0.125, DT[io], seqs=seqs)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("news,lens", [([1, 3], [100, 64]), ([40, 65], [100, 65]), ([1, 130], [300, 400])])
def test_values_that_are_not_finite_where_they_are_not_seen(io, news, lens):
    """Infinities and NaN in tokens that come after a query (or left its window) change nothing for it; who sees one has it."""
    print(f"case {io} {news} {lens}", flush=True)
    d, Hkv, H, window = 64, 1, 2, 30
    pool, rows = make(io, d, Hkv, 16, lens, 3)
    E, table = ref.per_group(DT[io]), pool.table.cpu()
    bad = {}                                                   # the last token but one of each sequence, and one a window before its end
    for s, m in enumerate(lens):
        for at, ch, x in ((m - 2, 5, float("inf")), (m - window - 2, 9, float("nan")), (m - 1, 63, -float("inf"))):
            p, slot = int(table[s, at // 16]), at % 16
            pool.v_pages[0, p, 0, slot // E, ch, slot % E] = x
            rows[s][1][at, 0, ch] = x
            bad[(s, at)] = ch
        p, slot = int(table[s, (m - 1) // 16]), (m - 1) % 16
        pool.k_pages[0, p, 0, 3, slot, 1] = float("nan")          # a key that is NaN: rows that see it are NaN
        rows[s][0][m - 1, 0, 3 * E + 1] = float("nan")
    q, start = queries(news, H, d, io, 4)
    out, lse = pool.attend(0, q, start, max_new=max(news), max_len=max(lens), window=window, want_lse=True)
    at = 0
    for s, (n, m) in enumerate(zip(news, lens)):
        got, x = ref.f64(out[at:at + n]), ref.f64(q[at:at + n])
        k, v = rows[s]
        for i in range(n):
            p = m - n + i
            seen = list(range(max(0, p - window + 1), p + 1))
            for h in range(H):
                if m - 1 in seen:
                    assert np.isnan(got[i, h]).all()
                    continue
                with np.errstate(invalid="ignore"):
                    want, _ = ref.attend(x[i:i + 1, h:h + 1], k[:p + 1], v[:p + 1], 0.125, window)
                    tol = ref.attend_bound(x[i:i + 1, h:h + 1], k[:p + 1], np.nan_to_num(v[:p + 1], nan=0.0, posinf=0.0, neginf=0.0), 0.125, DT[io], window)
                fine = np.isfinite(want[0, 0])
                assert (np.isfinite(got[i, h]) == fine).all(), (s, i, h)
                assert (np.abs(got[i, h] - want[0, 0])[fine] <= tol[0, 0][fine]).all()
                inf = np.isinf(want[0, 0])
                assert (got[i, h][inf] == want[0, 0][inf]).all()
        at += n


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 5, 70])
def test_pages_that_are_not_there(io, n):
    """Page numbers outside the pool: their tokens count as absent, and a row with none left gives zero."""
    lens = [200, 90, 150]
    pool, rows = make(io, 64, 2, 16, lens, 8)
    table = pool.table
    table[0, 3], table[0, 12], table[0, 0] = -1, pool.pages, 2 ** 31 - 1
    table[1, :] = -2 ** 31
    there = [np.ones(m, bool) for m in lens]
    for j in (3, 12, 0):
        there[0][16 * j:16 * j + 16] = False
    there[1][:] = False
    q, start = queries([n] * 3, 4, 64, io, 2)
    out, lse = pool.attend(0, q, start, max_new=n, max_len=200, want_lse=True)
    check(out, lse, q, [n] * 3, rows, 0.125, DT[io], there=there)
    assert (out[n:2 * n] == 0).all() and torch.isneginf(lse[n:2 * n]).all()
    # rows outside the table, lengths outside their rows
    pool.lens.copy_(torch.tensor([-5, 10 ** 9, 150], dtype=torch.int32))
    out, lse = pool.attend(0, q, start, torch.tensor([0, 99, 2], dtype=torch.int32, device="cuda"), max_new=n, max_len=200, want_lse=True)
    assert (out[:2 * n] == 0).all() and torch.isneginf(lse[:2 * n]).all()
    check(out[2 * n:], lse[2 * n:], q[2 * n:], [n], rows[2:], 0.125, DT[io])


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_large_and_small_scores(io):
    """Scores of hundreds, which only a maximum taken away keeps finite, and a scale of its own."""
    pool, rows = make(io, 64, 1, 64, [400, 400], 6, scale=12.0)
    q, start = queries([3, 40], 2, 64, io, 6, scale=12.0)
    for scale in (1.0, 0.02, 1e-6):
        out, lse = pool.attend(0, q, start, max_new=40, max_len=400, scale=scale, want_lse=True)
        check(out, lse, q, [3, 40], rows, scale, DT[io])


@pytest.mark.parametrize("n", [1, 40])
def test_strided_queries_other_streams_and_the_same_bits(n):
    pool, rows = make("bf16", 64, 2, 64, [500, 700], 1)
    wide = torch.randn(2 * n, 9, 64, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    q, start = wide[:, 2:6], torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    out = pool.attend(0, q, start, max_new=n, max_len=700)
    check(out, None, q, [n, n], rows, 0.125, torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        other = pool.attend(0, q, start, max_new=n, max_len=700, stream=side)
        side.synchronize()
        assert torch.equal(out, other)
    torch.cuda.current_stream().wait_stream(side)
    given = torch.empty(pool.attend_workspace_bytes(2, 2 * n, 4, n, 700) + 256, dtype=torch.uint8, device="cuda")
    into = torch.full_like(out, 7.0)
    assert torch.equal(pool.attend(0, q, start, max_new=n, max_len=700, ws=given, out=into), out) and torch.equal(into, out)


@pytest.mark.parametrize("n", [1, 70])
def test_the_widest_window_is_none(n):
    pool, rows = make("f32", 64, 1, 16, [300, 70], 2)
    q, start = queries([n, n], 4, 64, "f32", 5)
    want = pool.attend(0, q, start, max_new=n, max_len=300, want_lse=True)
    for window in (300, 2 ** 28, 2 ** 31 - 1):
        out, lse = pool.attend(0, q, start, max_new=n, max_len=300, window=window, want_lse=True)
        check(out, lse, q, [n, n], rows, 0.125, torch.float32)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_nothing_to_do():
    pool, _ = make("bf16", 64, 2, 16, [30, 5], 2)
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    none = torch.zeros(3, dtype=torch.int32, device="cuda")
    before = pool.book.clone()
    for start in (none, none[:1]):
        out, lse = pool.attend(0, q, start, want_lse=True)
        assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
        assert pool.append(0, q, q[:, :2], q[:, :2], start).shape == (0, 4, 64)
    pool.reserve(none[:0], none[:0])
    pool.fork(none[:0], none[:0])
    pool.free(none[:0])
    assert torch.equal(pool.book, before)


def test_rows_behind_the_last_sequence_are_left_alone():
    pool, rows = make("bf16", 64, 1, 16, [50, 60], 2)
    for n in (1, 40):
        q, start = queries([n, n], 4, 64, "bf16", 5)
        q = torch.cat((q, torch.full_like(q[:3], float("nan"))))
        out = torch.full_like(q, 9.0)
        pool.attend(0, q, start, max_new=n, max_len=60, out=out)
        assert (out[2 * n:] == 9.0).all()
        check(out[:2 * n], None, q[:2 * n], [n, n], rows, 0.125, torch.bfloat16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("news", [(1, 1), (40, 40), (1, 40), (300, 300), (300, 1), (0, 300)])
def test_rows_behind_the_last_sequence_are_left_alone_where_keys_are_split(d, news):
    """Few and many rows to join, of sequences with many parts, one part and none; what lies in the memory of the parts behind them is nobody's."""
    print(f"case d={d} news={news}", flush=True)
    pool, rows = make("bf16", d, 1, 64, [5000, 310], d)
    q, start = queries(news, 4, d, "bf16", 5)
    n = q.shape[0]
    q = torch.cat((q, torch.full_like(q[:1], float("nan")).expand(3, -1, -1)))
    for trash in (float("nan"), 1.0):
        junk = [torch.full((16 << 20,), trash, device="cuda") for _ in range(2)]     # freed: the workspace may get it
        del junk
        out = torch.full_like(q, 9.0)
        _, lse = pool.attend(0, q, start, max_new=max(news), max_len=5000, out=out, want_lse=True)
        assert (out[n:] == 9.0).all()
        check(out[:n], lse[:n], q[:n], news, rows, d ** -0.5, torch.bfloat16)


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes of keys: its last pages are found."""
    page, Hkv, d = 256, 8, 128
    P = (5 << 30) // (page * Hkv * d * 2)
    pool = binding.KvPages.empty(1, P, Hkv, d, page, 2, 4)
    g = torch.Generator(device="cuda").manual_seed(2)
    numbers = [P - 1, P - 3, P // 2 + 9, 0]
    for p in numbers:
        pool.k_pages[0, p].normal_(generator=g)
        pool.v_pages[0, p].normal_(generator=g)
    pool.table[1] = torch.tensor(numbers, dtype=torch.int32)
    pool.lens[1] = 1000
    k, v = (x[:1000] for x in ref.pool_rows(pool.k_pages[:, numbers].cpu(), pool.v_pages[:, numbers].cpu(), 0, [0, 1, 2, 3]))
    seqs = torch.tensor([1], dtype=torch.int32, device="cuda")
    for n in (1, 20):
        q, start = queries([n], 16, d, "bf16", n)
        out = pool.attend(0, q, start, seqs, max_new=n, max_len=1000)
        check(out, None, q, [n], [(ref.f64(k), ref.f64(v))], d ** -0.5, torch.bfloat16)
    row = torch.randn(40, 8 + 16, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    x = row[:, :8]
    pool.append(0, row[:, 8:], x, x, torch.tensor([0, 40], dtype=torch.int32, device="cuda"), seqs)
    k, v = (x[960:1000] for x in ref.pool_rows(pool.k_pages[:, numbers].cpu(), pool.v_pages[:, numbers].cpu(), 0, [0, 1, 2, 3]))
    assert torch.equal(k, x.cpu()) and torch.equal(v, x.cpu())
    src, dst = (torch.tensor([n], dtype=torch.int32, device="cuda") for n in (P - 1, P - 2))
    pool.copy(src, dst)
    assert torch.equal(pool.k_pages[0, P - 2], pool.k_pages[0, P - 1]) and torch.equal(pool.v_pages[0, P - 2], pool.v_pages[0, P - 1])


def test_a_captured_decode_loop():
    """Reserve, append and attend captured once and replayed token by token, with eager work between the replays, against eager calls of a second pool."""
    lens, H, Hkv, d, page = [30, 1, 90], 4, 2, 64, 16
    g = torch.Generator().manual_seed(11)
    pools = [binding.KvPages.empty(1, 40, Hkv, d, page, 3, 12) for _ in range(2)]
    seqs, one = torch.arange(3, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    start, rope = torch.arange(4, dtype=torch.int32, device="cuda"), binding.Rope.of(d)
    w = torch.ones(d, device="cuda")
    first = torch.tensor([0] + lens).cumsum(0).int().cuda()
    prompt = torch.randn(sum(lens), H + 2 * Hkv, d, generator=g).to(torch.bfloat16).cuda()
    outs = []
    for p in pools:
        p.reserve(seqs, torch.tensor(lens, dtype=torch.int32, device="cuda"))
        q = p.append(0, prompt[:, :H], prompt[:, H:H + Hkv], prompt[:, H + Hkv:], first, seqs, rope, w, w)
        outs.append(p.attend(0, q, first, seqs, max(lens), max(lens)))
    assert torch.equal(*outs)

    token = torch.empty(3, H + 2 * Hkv, d, dtype=torch.bfloat16, device="cuda")

    def step(p, x):
        p.reserve(seqs, one)
        q = p.append(0, x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], start, seqs, rope, w, w)
        return p.attend(0, q, start, seqs, 1, 190, want_lse=True)

    kept = pools[0].book.clone(), pools[0].k_pages.clone(), pools[0].v_pages.clone()
    token.copy_(prompt[:3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(pools[0], token)
        for x, y in zip((pools[0].book, pools[0].k_pages, pools[0].v_pages), kept):
            x.copy_(y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(pools[0], token)
    for t in range(40):
        token.copy_(torch.randn(3, H + 2 * Hkv, d, generator=g).to(torch.bfloat16))
        graph.replay()
        want, want_lse = step(pools[1], token)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), t
        assert torch.equal(pools[0].book, pools[1].book)
    assert torch.equal(pools[0].k_pages, pools[1].k_pages) and int(pools[0].status[0]) == 0
