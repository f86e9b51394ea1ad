"""Pages of 8 bits on the GPU against plain forms in 64 bits: append (codes, scales, blocks that fill), attention, and page management."""
import numpy as np
import pytest
import torch

import axes_ref
import e4m3_ref as ref
import paged_ref
from paper_2502_18394_amd import binding
from test_gpu_attend import FEW, MANY, MIXED, SHORT, SINGLES, check, queries
from test_gpu_heads import U32, _turn_size

pytestmark = pytest.mark.gpu
F8, BF16 = torch.float8_e4m3fn, torch.bfloat16
NAN = 0x7f


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _bits(pool):
    return pool.k_pages.view(torch.uint8).cpu().clone(), pool.v_pages.view(torch.uint8).cpu().clone(), pool.scales.cpu().clone()


# ---------------------------------------------------------------- append
def _append(pool, layer, rows, q, k, v, seqs, rope, w, eps=1e-6, **more):
    """One call with `rows[b]` tokens of each listed sequence, from the given rows [seq][token]."""
    start = torch.tensor([0] + [b - a for a, b in rows]).cumsum(0).int().cuda()
    part = lambda x: torch.cat([x[s][a:b] for s, (a, b) in zip(seqs, rows)])
    return pool.append(layer, part(q).cuda(), part(k).cuda(), part(v).cuda(), start, _ints(seqs), rope, *w, eps, **more)


def _check_block(pool, layer, row, first, n, calls, k64, size, v, d):
    """Tokens first .. first + n - 1 of one block, as `calls` (ends of the calls' tokens) wrote them: values from the plain form, bit for bit; keys within their roundings."""
    got_k, got_v, s = ref.rows(pool, layer, row, first + n)
    for h in range(pool.Hkv):
        scale_v, scale_k, codes, at = 0.0, 0.0, np.zeros((0, d), np.uint8), first
        border = False
        for end in calls + [first + n]:
            if end <= at:
                continue
            end = min(end, first + n)
            x = v[at:end, h]
            now = max(ref.scale_for(x), scale_v)
            codes = np.concatenate((ref.code(ref.numbers(torch.from_numpy(codes)).numpy() * (scale_v / now if at > first else 1.0)), ref.code(x / now)))
            y, off = k64[at:end, h], (d + 16) * U32 * size[at:end, h]
            low, high = ref.scale_for(np.abs(y) - off), ref.scale_for(np.abs(y) + off)
            border |= low != high
            scale_v, scale_k, at = now, max(high, scale_k), end
        assert s[first, h, 1] == scale_v
        assert np.array_equal(got_v[first:, h], ref.numbers(torch.from_numpy(codes)).numpy() * scale_v, equal_nan=True)
        assert s[first, h, 0] == scale_k or (border and s[first, h, 0] == scale_k / 2)
        want, off = k64[first:first + n, h], (d + 16) * U32 * size[first:first + n, h]
        # one rounding of the number, and codes below the smallest normal one rounded again as scales double: 2^-10 (1 + 1/2 + ...) of the last
        assert (np.abs(got_k[first:, h] - want) <= ref.STEP * np.abs(want) + 2 * ref.SMALL * s[first, h, 0] + 2 * off).all()


@pytest.mark.parametrize("page,d,H,Hkv", [(16, 64, 4, 2), (64, 64, 3, 3), (32, 128, 5, 1), (256, 128, 4, 4), (16, 64, 1, 1)])
@pytest.mark.parametrize("norm", [True, False])
def test_append(page, d, H, Hkv, norm):
    """Sequences that grow in calls of many sizes: new tokens in front of, at and behind the ends of blocks and pages; what is not theirs stays."""
    print(f"case page={page} d={d} H={H} Hkv={Hkv} norm={norm}", flush=True)
    g = torch.Generator().manual_seed(page + d + H)
    lens, seqs = [61, 16, 1, 33, 130], [3, 0, 5, 1, 2]
    ends = [[1, 2, 3, 17, 40, 41, 61], [16], [1], [15, 16, 32, 33], [0, 100, 130]]
    pool = binding.KvPages.empty(2, 70, Hkv, d, page, 6, 9, F8)
    noise = [torch.randint(0, 256, x.shape, generator=g, dtype=torch.uint8) for x in _bits(pool)[:2]]
    pool.k_pages.view(torch.uint8).copy_(noise[0])
    pool.v_pages.view(torch.uint8).copy_(noise[1])
    pool.scales.copy_(torch.exp2(torch.randint(-9, 9, pool.scales.shape, generator=g).float()))
    before = _bits(pool)
    rows = {s: n for s, n in zip(seqs, lens)}
    q, k, v = ({s: torch.randn(n, heads, d, generator=g).mul(torch.exp2(2 * torch.randn(n, 1, 1, generator=g))).to(BF16) for s, n in rows.items()} for heads in (H, Hkv, Hkv))
    rope = binding.Rope.of(d, 500000.0)
    w = [(1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in "qk"] if norm else [None, None]
    at, out = {s: 0 for s in seqs}, {s: [] for s in seqs}
    for step in range(max(map(len, ends))):
        part = [(s, at[s], e[step]) for s, e in zip(seqs, ends) if step < len(e)]
        pool.reserve(_ints([s for s, _, _ in part]), _ints([b - a for _, a, b in part]))
        got = _append(pool, 1, [(a, b) for _, a, b in part], q, k, v, [s for s, _, _ in part], rope, w)
        for s, a, b in part:
            out[s].append(got[:b - a])
            got = got[b - a:]
            at[s] = b
    assert int(pool.status[0]) == 0
    freq = paged_ref.f64(rope.inv_freq)
    written = torch.zeros(pool.pages, page, dtype=torch.bool)
    for s, e in zip(seqs, ends):
        n = rows[s]
        pos = np.arange(n)
        one = binding.qk_norm_rotate(q[s].cuda(), k[s].cuda(), None, rope, *w)
        assert torch.equal(torch.cat(out[s]), one[0])
        wk = None if w[1] is None else paged_ref.f64(w[1])
        plain = paged_ref.heads(k[s].double().numpy(), wk, pos, np.zeros(0), 1e-6)
        k64, size = paged_ref.heads(k[s].double().numpy(), wk, pos, freq, 1e-6), _turn_size(plain, d // 2, False)
        for first in range(0, n, 16):
            _check_block(pool, 1, s, first, min(16, n - first), [x for x in e if first < x < first + 16], k64, size, v[s].double().numpy(), d)
        for t in range(n):
            written[pool.table[s, t // page], t % page] = True
    # all that is no token's is as it was
    k_now, v_now, s_now = _bits(pool)
    assert all(torch.equal(a[0], b[0]) for a, b in zip((k_now, v_now, s_now), before))
    gone = ~written
    a, b = (x[1].permute(0, 3, 1, 2, 4)[gone] for x in (k_now, before[0]))
    assert torch.equal(a, b)
    a, b = (x[1].permute(0, 2, 4, 1, 3).reshape(pool.pages, page, Hkv, d)[gone] for x in (v_now, before[1]))
    assert torch.equal(a, b)
    blocks = ~written.view(pool.pages, page // 16, 16).any(-1)
    a, b = (x[1].permute(0, 2, 1, 3)[blocks] for x in (s_now, before[2]))
    assert torch.equal(a, b)


def test_numbers_at_the_ends_of_the_range():
    """Blocks of zeros, of tiny and of the largest numbers, with infinities and NaN among them."""
    pool = binding.KvPages.empty(1, 8, 1, 64, 16, 1, 8, F8)
    v = torch.zeros(96, 1, 64, dtype=BF16)
    v[16:32] = torch.linspace(-1, 1, 64).to(BF16) * 2.0 ** -60
    v[32:48] = 3.3895e38
    v[32, 0, 0], v[33, 0, 0] = -3.3895e38, 1.0
    v[48:64] = torch.linspace(-3, 3, 64).to(BF16)
    v[50, 0, 3], v[51, 0, 4], v[52, 0, 5] = float("inf"), float("-inf"), float("nan")
    v[64:80], v[80:96] = float("nan"), 2.0 ** -120
    v[80, 0, 0] = 448 * 2.0 ** -101
    pool.reserve(_ints([0]), _ints([96]))
    pool.append(0, v.cuda(), v.cuda(), v.cuda(), _ints([0, 96]))
    k_got, v_got, s = ref.rows(pool, 0, 0, 96)
    assert np.array_equal(k_got, v_got, equal_nan=True) and (s[..., 0] == s[..., 1]).all()
    x = v.double().numpy()
    assert (s[0] == 2.0 ** -100).all() and (v_got[:16] == 0).all()
    assert s[16, 0, 1] == ref.scale_for(x[16:32]) and (np.abs(v_got[16:32] - x[16:32]) <= ref.STEP * np.abs(x[16:32]) + ref.SMALL * s[16, 0, 1]).all()
    assert s[32, 0, 1] == 2.0 ** 120 and np.abs(v_got[32:48]).max() == 1.875 * 2.0 ** 127 and v_got[32, 0, 0] < 0 and v_got[33, 0, 0] == 0
    fine = np.isfinite(x[48:64])
    assert np.array_equal(np.isfinite(v_got[48:64]), fine) and fine.sum() == 16 * 64 - 3
    assert (np.abs(v_got[48:64] - x[48:64])[fine] <= (ref.STEP * np.abs(x[48:64]) + ref.SMALL * s[48, 0, 1])[fine]).all()
    assert np.isnan(v_got[64:80]).all() and s[64, 0, 1] == 2.0 ** -100
    assert s[80, 0, 1] == 2.0 ** -100 and v_got[80, 0, 0] == x[80, 0, 0] and (v_got[81:] == 0).all()
    # the largest finite number stays finite where it is attended over
    pool.free(_ints([0]))
    pool.reserve(_ints([0]), _ints([33]))
    pool.append(0, v[:33].cuda(), torch.zeros_like(v[:33]).cuda(), v[:33].cuda(), _ints([0, 33]))
    out = pool.attend(0, torch.zeros(33, 1, 64, dtype=BF16, device="cuda"), _ints([0, 33]), max_new=33, max_len=33)
    assert torch.isfinite(out).all() and out[32].abs().max() > 1e36


def test_append_leaves_out_what_has_no_place():
    """A page that is outside the pool, a page of two users, a row outside the table, a failed reserve: queries at most, never a byte of the pool."""
    g = torch.Generator().manual_seed(2)
    pool = binding.KvPages.empty(1, 6, 2, 64, 16, 3, 4, F8)
    x = torch.randn(4, 2, 64, generator=g).to(BF16).cuda()
    pool.reserve(_ints([0, 1]), _ints([18, 18]))
    start = _ints([0, 2, 4])
    before = _bits(pool)
    for change in ("outside", "shared", "row", "status"):
        book = pool.book.clone()
        seqs = [0, 1]
        if change == "outside":
            pool.table[0, 1], pool.table[1, 1] = 6, -5
        elif change == "shared":
            pool.refs[pool.table[0, 1].long()] = 2
            pool.refs[pool.table[1, 1].long()] = 2
        elif change == "row":
            seqs = [7, -1]
        else:
            pool.status[0] = pool.NO_PAGES
        pool.append(0, x, x, x, start, _ints(seqs))
        assert all(torch.equal(a, b) for a, b in zip(_bits(pool), before)), change
        assert int(pool.status[0]) == {"shared": pool.SHARED, "status": pool.NO_PAGES}.get(change, 0)
        pool.book.copy_(book)


# ---------------------------------------------------------------- attention
def make(d, Hkv, page, lens, seed, layers=1, fill=NAN):
    """A pool whose sequences hold random codes with random scales, everything else NaN; with the keys and values, [m, Hkv, d] each."""
    g = torch.Generator().manual_seed(seed)
    M, P = max(1, max(-(-n // page) for n in lens)) + 1, sum(-(-n // page) for n in lens) + 4
    pool = binding.KvPages.empty(layers, P, Hkv, d, page, len(lens), M, F8)
    order, layer = torch.randperm(P, generator=g), layers - 1
    table, refs, at = pool.table.cpu(), pool.refs.cpu(), 0
    coded = lambda *shape: (torch.randn(*shape, generator=g) * 90).clamp(-448, 448).to(F8).view(torch.uint8)
    k, v = coded(P, page, Hkv, d), coded(P, page, Hkv, d)
    power = torch.randint(-8, -5, (P, Hkv, page // 16, 2), generator=g)
    live = torch.zeros(P, page, dtype=torch.bool)
    for s, n in enumerate(lens):
        m = -(-n // page)
        mine = order[at:at + m]
        at += m
        table[s, :m], refs[mine] = mine.int(), 1
        for i in range(n):
            live[mine[i // page], i % page] = True
    k[~live], v[~live] = fill, fill | 0x80
    pool.k_pages.view(torch.uint8).fill_(fill)
    pool.v_pages.view(torch.uint8).fill_(fill)
    pool.k_pages.view(torch.uint8)[layer] = k.view(P, page, Hkv, d // 16, 16).permute(0, 2, 3, 1, 4).cuda()
    pool.v_pages.view(torch.uint8)[layer] = v.view(P, page // 16, 16, Hkv, d).permute(0, 3, 1, 4, 2).cuda()
    pool.scales[layer] = torch.exp2(power.float()).cuda()
    pool.table.copy_(table)
    pool.refs.copy_(refs)
    pool.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return pool, [ref.rows(pool, layer, s, n)[:2] for s, n in enumerate(lens)]


@pytest.mark.parametrize("d,page", [(64, 16), (64, 64), (64, 256), (128, 32), (128, 128)])
@pytest.mark.parametrize("H,Hkv", [(4, 1), (2, 2), (7, 1)])
@pytest.mark.parametrize("name", ["SINGLES", "FEW", "MANY", "MIXED", "SHORT"])
def test_attention_against_the_definition(d, page, H, Hkv, name):
    print(f"case {name} d={d} page={page} H={H} Hkv={Hkv}", flush=True)
    news, lens = {"SINGLES": SINGLES, "FEW": FEW, "MANY": MANY, "MIXED": MIXED, "SHORT": SHORT}[name]
    pool, rows = make(d, Hkv, page, lens, d + page + H)
    q, start = queries(news, H, d, "bf16", H)
    out, lse = pool.attend(0, q, start, max_new=max(news), max_len=max(lens), want_lse=True)
    check(out, lse, q, news, rows, d ** -0.5, BF16)


@pytest.mark.parametrize("window", [1, 7, 64, 100])
@pytest.mark.parametrize("name", ["SINGLES", "FEW", "MANY", "MIXED"])
def test_windows(window, name):
    print(f"case {name} window={window}", flush=True)
    news, lens = {"SINGLES": SINGLES, "FEW": FEW, "MANY": MANY, "MIXED": MIXED}[name]
    pool, rows = make(64, 2, 16, lens, window)
    q, start = queries(news, 4, 64, "bf16", window)
    out, lse = pool.attend(0, q, start, max_new=max(news), max_len=max(lens), window=window, want_lse=True)
    check(out, lse, q, news, rows, 0.125, BF16, window)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 4, 9, 17, 60, 300])
def test_keys_split_over_workgroups(d, n):
    """One sequence of many keys: its keys are divided, and the parts joined."""
    print(f"case d={d} n={n}", flush=True)
    pool, rows = make(d, 2, 32, [2900], d + n)
    q, start = queries([n], 4, d, "bf16", n)
    out, lse = pool.attend(0, q, start, max_new=n, max_len=2900, want_lse=True)
    check(out, lse, q, [n], rows, d ** -0.5, BF16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 4, 7, 8])
@pytest.mark.parametrize("rows", [17, 32, 33, 48, 49, 64, 65])
def test_some_rows_of_a_key_head(d, G, rows):
    """Several new tokens of a few sequences, from one group of 16 rows of a key head to the first tile: sequences with fewer, one and no tokens, more new tokens than
    there are tokens, with a window and without."""
    print(f"case d={d} G={G} rows={rows}", flush=True)
    n = rows // G
    news, lens = [n, 1, 0, n, n // 2 + 1, n], [n + 700, 90, 5, n, 64, max(1, n - 2)]
    page = (16, 256)[rows % 2]
    pool, kv = make(d, 2, page, lens, d + G + rows)
    q, start = queries(news, 2 * G, d, "bf16", rows)
    for window in (0, 50):
        out, lse = pool.attend(0, q, start, max_new=n, max_len=max(lens), window=window, want_lse=True)
        check(out, lse, q, news, kv, d ** -0.5, BF16, window)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [5, 11, 16])
def test_some_rows_with_absent_pages_and_nan(d, n):
    """As above, four rows a token: absent pages hide their tokens, a NaN value reaches the rows that see it and no other."""
    print(f"case d={d} n={n}", flush=True)
    m, H = 700, 4
    pool, kv = make(d, 1, 16, [m, m], n)
    there = np.ones(m, bool)
    for j, value in ((0, -1), (3, pool.pages), (20, -7), (43, 1 << 30)):
        pool.table[0, j] = value
        there[16 * j:16 * j + 16] = False
    q, start = queries([n, n], H, d, "bf16", 5)
    out, lse = pool.attend(0, q, start, max_new=n, max_len=m, want_lse=True)
    check(out, lse, q, [n, n], kv, d ** -0.5, BF16, there=[there, np.ones(m, bool)])
    at, channel = m - n + 2, 5                                # all tokens but the first two see it
    pool.v_pages.view(torch.uint8)[0, int(pool.table[1, at // 16]), 0, 0, channel, at % 16] = NAN
    got = pool.attend(0, q, start, max_new=n, max_len=m).float().cpu()
    bad = torch.zeros(2 * n, H, d, dtype=torch.bool)
    bad[n + 2:, :, channel] = True
    assert torch.equal(got.isnan(), bad) and torch.equal(got[~bad], out.float().cpu()[~bad])


@pytest.mark.parametrize("d", [64, 128])
def test_some_rows_that_the_call_is_not_sized_for(d):
    """A sequence with more new tokens than max_new says, and rows behind the last sequence, stay as they are; the others are the same without them."""
    news, lens, H = [8, 9, 3], [300, 1200, 70], 4
    pool, kv = make(d, 1, 64, lens, d)
    q, start = queries(news + [4], H, d, "bf16", 1)
    out = torch.full_like(q, 7)
    lse = torch.full((q.shape[0], H), 7.0, device="cuda")
    pool.attend(0, q, start[:4].contiguous(), max_new=8, max_len=1200, out=out, lse=lse)
    for t in (out, lse):
        assert (t[8:17] == 7).all() and (t[20:] == 7).all()
    check(torch.cat((out[:8], out[17:20])), torch.cat((lse[:8], lse[17:20])), torch.cat((q[:8], q[17:20])), [8, 3], [kv[0], kv[2]], d ** -0.5, BF16)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n", [1, 40])
def test_pages_that_are_absent_and_values_that_are_nan(page, n):
    """Pages outside the pool hide their tokens; a NaN value reaches the rows that see it and no other."""
    print(f"case page={page} n={n}", flush=True)
    m = 150
    pool, rows = make(64, 1, page, [m], 7 + page)
    q, start = queries([n], 3, 64, "bf16", 5)
    there = np.ones(m, bool)
    for j in (0, 1):
        pool.table[0, j] = (-1, pool.pages + 3)[j]
        there[j * page:(j + 1) * page] = False
    out, lse = pool.attend(0, q, start, max_new=n, max_len=m, want_lse=True)
    check(out, lse, q, [n], rows, 0.125, BF16, there=[there])
    if n == 1:
        return
    at, channel = m - 20, 5                                  # the last 20 rows see it
    number, slot = int(pool.table[0, at // page]), at % page
    pool.v_pages.view(torch.uint8)[0, number, 0, slot // 16, channel, slot % 16] = NAN
    got = pool.attend(0, q, start, max_new=n, max_len=m).float().cpu()
    bad = torch.zeros(n, 3, 64, dtype=torch.bool)
    bad[n - 20:, :, channel] = True
    assert torch.equal(got.isnan(), bad) and torch.equal(got[~bad], out.float().cpu()[~bad])


def test_the_same_numbers_as_a_pool_of_bf16():
    """Codes times scales are bf16 numbers: a bf16 pool that holds them gives the same outputs, but for the order of the sums."""
    pool, rows = make(64, 2, 64, [700, 90], 3)
    other = binding.KvPages.empty(1, pool.pages, 2, 64, 64, 2, pool.max_pages)
    other.book.copy_(pool.book)
    s = pool.scales.repeat_interleave(16, 3)                 # [layers, pages, Hkv, page, 2]
    k = (pool.k_pages.float() * s[:, :, :, None, :, 0, None]).permute(0, 1, 2, 4, 3, 5).reshape(1, pool.pages, 2, 64, 64)
    v = (pool.v_pages.float().permute(0, 1, 2, 3, 5, 4).reshape(1, pool.pages, 2, 64, 64) * s[..., 1, None])
    assert torch.equal(k.bfloat16().float().nan_to_num(), k.nan_to_num())
    other.k_pages.copy_(k.view(1, pool.pages, 2, 64, 8, 8).permute(0, 1, 2, 4, 3, 5))
    other.v_pages.copy_(v.view(1, pool.pages, 2, 8, 8, 64).permute(0, 1, 2, 3, 5, 4))
    for news in ([1, 1], [200, 50]):
        q, start = queries(news, 4, 64, "bf16", 1)
        a, b = (x.attend(0, q, start, max_new=max(news), max_len=700, want_lse=True) for x in (pool, other))
        at = 0
        for n, (kk, vv) in zip(news, rows):
            tol = paged_ref.attend_bound(paged_ref.f64(q[at:at + n]), kk, vv, 0.125, BF16)
            assert (np.abs(paged_ref.f64(a[0][at:at + n]) - paged_ref.f64(b[0][at:at + n])) <= 2 * tol).all()
            at += n


def test_layers_strides_and_streams():
    """The last of three layers, queries with something between the tokens, another stream than the current one, a given workspace; rows behind the last sequence stay."""
    pool, rows = make(64, 2, 32, [90, 300], 11, layers=3)
    wide = torch.randn(8, 6, 64).to(BF16).cuda()
    q, start = wide[:, 1:5], _ints([0, 2, 5])
    out, lse = torch.full((8, 4, 64), 7.0, dtype=BF16, device="cuda"), torch.full((8, 4), 7.0, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(pool.attend_workspace_bytes(2, 8, 4, 3, 300) + 256, dtype=torch.uint8, device="cuda")
    pool.attend(2, q, start, max_new=3, max_len=300, out=out, lse=lse, ws=ws, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    check(out, lse, q, [2, 3], rows, 0.125, BF16)
    assert (out[5:] == 7).all() and (lse[5:] == 7).all()


# ---------------------------------------------------------------- pages, and all of it together
@pytest.mark.parametrize("page,d,Hkv", [(16, 64, 2), (64, 128, 3), (256, 64, 1)])
def test_scales_go_with_their_pages(page, d, Hkv):
    print(f"case page={page} d={d} Hkv={Hkv}", flush=True)
    g = torch.Generator().manual_seed(page)
    pool = binding.KvPages.empty(2, 37, Hkv, d, page, 9, 8, F8)
    book = paged_ref.Book(9, 37, 8, page)
    for x in (pool.k_pages, pool.v_pages):
        x.view(torch.uint8).copy_(torch.randint(0, 256, x.shape, generator=g, dtype=torch.uint8))
    pool.scales.copy_(torch.rand(pool.scales.shape, generator=g))
    k, v, s = _bits(pool)

    def same():
        assert pool.book.tolist() == book.words()
        assert all(torch.equal(a, b) for a, b in zip(_bits(pool), (k, v, s)))

    def fork(src, dst):
        pool.fork(_ints(src), _ints(dst))
        for a, b, rest in book.fork(src, dst):
            some = -(-rest // 16)
            k[:, b, :, :, :16 * some] = k[:, a, :, :, :16 * some]
            v[:, b, :, :some] = v[:, a, :, :some]
            s[:, b, :, :some] = s[:, a, :, :some]

    seqs, add = [4, 0, 7], [page * 3 + 5, 1, 0]
    pool.reserve(_ints(seqs), _ints(add))
    book.reserve(seqs, add)
    fork([4, 0, 0, 7], [1, 2, 8, 3])
    same()
    pool.free(_ints([4, 2]))
    book.free([4, 2])
    pool.compact()
    for a, b in book.compact():
        k[:, b], v[:, b], s[:, b] = k[:, a], v[:, a], s[:, a]
    same()
    pool.copy(_ints([0, 30, 2]), _ints([36, 31, 20]))
    for a, b in ((0, 36), (30, 31), (2, 20)):
        k[:, b], v[:, b], s[:, b] = k[:, a], v[:, a], s[:, a]
    same()


def test_a_decode_loop_captured():
    """Reserve, append and attend of three sequences in one graph, replayed token by token with eager work between, against a pool that is worked on eagerly."""
    g = torch.Generator().manual_seed(5)
    lens = [5, 31, 64]
    pools = [binding.KvPages.empty(1, 40, 2, 64, 16, 3, 12, F8) for _ in range(2)]
    rope, seqs, one = binding.Rope.of(64), _ints([0, 1, 2]), _ints([1, 1, 1])
    prompt = [torch.randn(sum(lens), n, 64, generator=g).to(BF16).cuda() for n in (4, 2, 2)]
    for pool in pools:
        pool.reserve(seqs, _ints(lens))
        pool.append(0, *prompt, _ints([0, 5, 36, 100]), seqs, rope)
    rows = [torch.zeros(3, n, 64, dtype=BF16, device="cuda") for n in (4, 2, 2)]
    start = _ints([0, 1, 2, 3])

    def step(pool):
        pool.reserve(seqs, one)
        q = pool.append(0, *rows, start, seqs, rope)
        return q, pool.attend(0, q, start, seqs, 1, 192, want_lse=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    state = [x.clone() for x in (pools[0].book, pools[0].k_pages, pools[0].v_pages, pools[0].scales)]
    with torch.cuda.stream(side):
        step(pools[0])
        for a, b in zip((pools[0].book, pools[0].k_pages, pools[0].v_pages, pools[0].scales), state):
            a.copy_(b)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(pools[0])
    for i in range(20):
        for x in rows:
            x.copy_((torch.randn(x.shape, generator=g) * (1 + i % 5)).to(BF16))
        graph.replay()
        want = step(pools[1])
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1][0], want[1][0]) and torch.equal(got[1][1], want[1][1]), i
        assert all(torch.equal(a, b) for a, b in zip(_bits(pools[0]), _bits(pools[1]))), i
    # and it is attention over what the blocks hold
    for b, n in enumerate(lens):
        k, v, _ = ref.rows(pools[1], 0, b, n + 20)
        check(want[1][0][b:b + 1], want[1][1][b:b + 1], want[0][b:b + 1], [1], [(k, v)], 0.125, BF16)


def test_tokens_one_by_one_end_as_all_at_once():
    """A block that fills token by token has the scale of one that came at once, and the same codes but for subnormal ones that were rounded at a smaller scale first."""
    g = torch.Generator().manual_seed(8)
    v = (torch.randn(37, 2, 64, generator=g) * torch.exp2(2 * torch.randn(37, 1, 1, generator=g))).to(BF16).cuda()
    pools = [binding.KvPages.empty(1, 8, 2, 64, 32, 1, 8, F8) for _ in range(2)]
    pools[0].reserve(_ints([0]), _ints([37]))
    pools[0].append(0, v, v, v, _ints([0, 37]))
    for i in range(37):
        pools[1].reserve(_ints([0]), _ints([1]))
        pools[1].append(0, v[i:i + 1], v[i:i + 1], v[i:i + 1], _ints([0, 1]))
    (ka, va, sa), (kb, vb, sb) = (ref.rows(p, 0, 0, 37) for p in pools)
    assert np.array_equal(sa, sb)
    for a, b, s in ((ka, kb, sa[..., :1]), (va, vb, sa[..., 1:])):
        normal = np.abs(a) >= 2.0 ** -5 * s
        assert np.array_equal(a[normal], b[normal]) and (np.abs(a - b) <= 2 * ref.SMALL * s * np.ones_like(a)).all()


def test_pages_beyond_four_gigabytes():
    """A pool whose keys alone are more than 2^32 bytes: the last pages are written, read, forked and copied where they lie, and nothing in front of them."""
    pages, Hkv, page, d = 33000, 8, 256, 64                  # 4.3 GB of keys
    pool = binding.KvPages.empty(1, pages, Hkv, d, page, 3, 4, F8)
    last = [pages - 1, pages - 2, pages - 3]
    pool.table[0, :3] = _ints(last)
    pool.refs[_ints(last).long()] = 1
    pool.lens[0] = 600
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(600, n, d, generator=g).to(BF16).cuda() for n in (16, Hkv, Hkv))
    pool.append(0, q, k, v, _ints([0, 600]), _ints([0]))
    assert not pool.k_pages.view(torch.uint8)[0, :pages - 3].any() and not pool.v_pages.view(torch.uint8)[0, :pages - 3].any()
    k_got, v_got, s = ref.rows(Window(pool, pages - 3), 0, 0, 600)
    rows, x = [(k_got, v_got)], v.double().cpu().numpy()
    assert (np.abs(v_got - x) <= ref.STEP * np.abs(x) + ref.SMALL * s[..., 1:]).all()          # half a step of a normal number, or of a subnormal one: 2^-10 of the scale
    for n in (1, 40):
        out, lse = pool.attend(0, q[:n].contiguous(), _ints([0, n]), _ints([0]), n, 600, want_lse=True)
        check(out, lse, q[:n], [n], rows, 0.125, BF16)
    pool.fork(_ints([0]), _ints([1]))                        # the last page goes to page 0
    pool.copy(_ints([pages - 1]), _ints([pages - 5]))
    assert pool.table[1, :3].tolist() == [pages - 1, pages - 2, 0] and int(pool.status[0]) == 0
    # whole groups of 16 tokens: 600 - 512 = 88 are 96
    assert torch.equal(pool.k_pages.view(torch.uint8)[0, 0, :, :, :96], pool.k_pages.view(torch.uint8)[0, pages - 3, :, :, :96])
    assert torch.equal(pool.scales[0, 0, :, :6], pool.scales[0, pages - 3, :, :6]) and (pool.scales[0, 0, :, 6:] == 1).all()
    for x in (pool.k_pages, pool.v_pages, pool.scales):
        assert torch.equal(x.view(torch.uint8)[0, pages - 5], x.view(torch.uint8)[0, pages - 1])


class Window:
    """The pages from `first` on of a pool, as e4m3_ref.rows looks at one."""

    def __init__(self, pool, first):
        self.page, self.Hkv, self.d = pool.page, pool.Hkv, pool.d
        self.table = (pool.table - first).clamp(min=-1)
        self.k_pages, self.v_pages, self.scales = (x.view(torch.uint8)[:, first:].contiguous().view(x.dtype) for x in (pool.k_pages, pool.v_pages, pool.scales))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rot,interleaved,axes", [(32, False, 1), (32, True, 1), (0, False, 1), (None, True, 1), (None, False, 3), (None, True, 2), (48, False, 8)])
def test_append_with_every_way_of_turning(d, rot, interleaved, axes):
    """Part of a row, adjacent pairs, no rotation, several axes, positions given for one; rows of one projection, with something between the tokens; rows behind the last sequence stay."""
    rot = d if rot is None else rot
    print(f"case d={d} rot={rot} interleaved={interleaved} axes={axes}", flush=True)
    H, Hkv, news, had, seqs, page = 5, 3 if d == 64 else 1, [21, 1, 40], [10, 5, 0], [1, 0, 2], 32
    H *= Hkv
    T, g = sum(news), torch.Generator().manual_seed(d + rot + axes)
    pool = binding.KvPages.empty(1, 12, Hkv, d, page, 3, 4, F8)
    pool.reserve(_ints(seqs), _ints(had))
    pool.append(0, *(torch.zeros(sum(had), n, d, dtype=BF16, device="cuda") for n in (H, Hkv, Hkv)), _ints([0, 10, 15, 15]), _ints(seqs))     # blocks of zeros, the least scale
    pool.reserve(_ints(seqs), _ints(news))
    wide = torch.randn(T + 3, H + 2 * Hkv + 1, d, generator=g).to(BF16).cuda()
    q, k, v = wide[:, :H], wide[:, H:H + Hkv], wide[:, H + Hkv:H + 2 * Hkv]
    axis = torch.cat((torch.arange(axes), torch.randint(0, axes, (max(rot // 2 - axes, 0),), generator=g))) if rot else None
    rope = binding.Rope.of(rot, 500000.0, interleaved, axes=axis if axes > 1 else None) if rot else None
    places = torch.cat([torch.arange(a, a + n) for n, a in zip(news, had)] + [torch.zeros(3, dtype=torch.long)])
    pos = torch.randint(0, 90000, (axes, T + 3), generator=g, dtype=torch.int32) if axes > 1 or rot == 32 else places[None].int()
    w = [(1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in "qk"]
    out = torch.full((T + 3, H, d), 7.0, dtype=BF16, device="cuda")
    given = pos.cuda() if axes > 1 or rot == 32 else None
    pool.append(0, q, k, v, torch.tensor([0] + news).cumsum(0).int().cuda(), _ints(seqs), rope, *w, 1e-6, out, positions=given)
    assert (out[T:] == 7).all() and int(pool.status[0]) == 0
    both = binding.qk_norm_rotate(q, k, pos.cuda() if axes > 1 else pos[0].cuda(), rope, *w)
    assert torch.equal(out[:T], both[0][:T])
    freq = paged_ref.f64(rope.inv_freq) if rot else np.zeros(0)
    angle = axes_ref.angles(pos.numpy(), axis.numpy() if axes > 1 else np.zeros(rot // 2, int), freq) if rot else np.zeros((T + 3, 0))
    plain = axes_ref.heads(k.double().cpu().numpy(), paged_ref.f64(w[1]), angle * 0, 1e-6, interleaved)
    k64, size, v64 = axes_ref.heads(k.double().cpu().numpy(), paged_ref.f64(w[1]), angle, 1e-6, interleaved), _turn_size(plain, rot // 2, interleaved), v.double().cpu().numpy()
    at = 0
    for s, n, before in zip(seqs, news, had):
        zeros = np.zeros((before, Hkv, d))
        rows = [np.concatenate((zeros, x[at:at + n])) for x in (k64, size, v64)]
        for first in range(0, before + n, 16):
            _check_block(pool, 0, s, first, min(16, before + n - first), [before] if first < before < first + 16 else [], *rows, d)
        at += n
