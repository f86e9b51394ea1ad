"""Norm and rotation of query and key heads on the GPU against the 64-bit form: values, gradients, gradients against differences, pages."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2502_18394_amd import binding

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U32 = 2.0 ** -24


def _inputs(T, H, Hkv, d, io, seed, fused=False):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).to(DT[io]).cuda()
    if fused:                                            # heads of one projection's rows, with something between the tokens
        row = torch.randn(T, H + 2 * Hkv + 1, d, generator=g).to(DT[io]).cuda()
        q, k = row[:, :H], row[:, H:H + Hkv]
    else:
        q, k = r(T, H, d), r(T, Hkv, d)
    w = [(1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in "qk"]
    return q, k, w, g


def _turn_size(y, half, interleaved):
    """|a| + |b| of each channel's pair."""
    a = np.abs(np.array(y, np.float64))
    out = a.copy()
    if half:
        i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        out[..., i] = out[..., j] = a[..., i] + a[..., j]
    return out


def _check(got, want, size, dtype, d):
    """One rounding to the type, and 32-bit arithmetic: a sum of d squares, a root, three products, a turn."""
    err = np.abs(ref.f64(got) - want)
    tol = ref.half_step(dtype) * np.abs(want) + (d + 16) * U32 * size
    assert np.isfinite(ref.f64(got)).all() and (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())


CASES = [  # T, H, Hkv, d, rot, interleaved, norm, fused
    (1, 1, 1, 64, 64, False, True, False), (1, 32, 8, 64, 64, False, True, False), (7, 5, 5, 64, 64, True, True, True),
    (8, 4, 2, 128, 128, False, True, True), (9, 3, 1, 128, 32, False, True, False), (17, 7, 7, 64, 16, True, True, False),
    (130, 12, 4, 64, 0, False, True, False), (33, 6, 2, 128, 128, True, False, True), (5, 2, 1, 64, 48, False, False, False),
    (1003, 32, 8, 64, 64, False, True, True), (0, 4, 2, 64, 64, False, True, False),
]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,Hkv,d,rot,interleaved,norm,fused", CASES)
def test_forward_and_backward(T, H, Hkv, d, rot, interleaved, norm, fused, io):
    print(f"case T={T} H={H} Hkv={Hkv} d={d} rot={rot} interleaved={interleaved} norm={norm} {io}", flush=True)
    q, k, w, g = _inputs(T, H, Hkv, d, io, T + d + rot, fused)
    pos = torch.randint(0, 1 << 20, (T,), generator=g, dtype=torch.int32)
    if T > 2:
        pos[0], pos[1], pos[2] = 0, 2 ** 31 - 1, 131071
    rope = binding.Rope.of(rot, 500000.0, interleaved) if rot else None
    freq = ref.f64(rope.inv_freq) if rot else np.zeros(0)
    wq, wk = w if norm else (None, None)
    got = binding.qk_norm_rotate(q, k, pos.cuda(), rope, wq, wk, 1e-5)
    dy = [torch.randn(x.shape, generator=g).to(DT[io]).cuda() for x in (q, k)]
    grads = binding.qk_norm_rotate_backward(*dy, q, k, pos.cuda(), rope, wq, wk, 1e-5)
    for n, (x, weight, y) in enumerate(((q, wq, got[0]), (k, wk, got[1]))):
        x64, w64 = ref.f64(x), None if weight is None else ref.f64(weight)
        plain = ref.heads(x64, w64, pos, np.zeros(0), 1e-5)
        _check(y, ref.heads(x64, w64, pos, freq, 1e-5, interleaved), _turn_size(plain, rot // 2, interleaved), DT[io], d)
        d64 = ref.f64(dy[n])
        want, want_w = ref.heads_backward(d64, x64, w64, pos, freq, 1e-5, interleaved)
        size = _turn_size(d64, rot // 2, interleaved)
        if norm:
            r = 1 / np.sqrt((x64 * x64).mean(-1, keepdims=True) + 1e-5)
            h, xh = size * np.abs(w64), np.abs(x64 * r)
            _check(grads[n], want, 3 * r * (h + xh * (h * xh).mean(-1, keepdims=True)), DT[io], d)
            # products and the sums of one run of 8 tokens in 32 bits (at most 8 H terms), the rest in 64, one rounding
            tol = (d + 16 + 8 * H) * U32 * (size * xh).sum((0, 1)) + U32 * np.abs(want_w) + 1e-300
            assert (np.abs(ref.f64(grads[2 + n]) - want_w) <= tol).all()
        else:
            _check(grads[n], want, size, DT[io], d)
            assert grads[2 + n] is None


def test_default_positions_and_no_rotation_are_exact_copies():
    q, k, _, _ = _inputs(11, 3, 2, 64, "bf16", 5)
    got = binding.qk_norm_rotate(q, k)
    assert torch.equal(got[0], q) and torch.equal(got[1], k)
    rope = binding.Rope.of(64)
    a = binding.qk_norm_rotate(q, k, None, rope)
    b = binding.qk_norm_rotate(q, k, torch.arange(11, dtype=torch.int32, device="cuda"), rope)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_against_differences(interleaved):
    """The slope of sum(dy * y) along a direction, from the GPU's fp32 forward pass at x +- h u: the difference's own error is h^2 / 6 of the third
    derivative (below 1e-4 of the slope's size here) and 2 * 2^-24 sqrt(terms) |dy y| / h of rounding."""
    T, H, Hkv, d = 6, 3, 2, 64
    q, k, (wq, wk), g = _inputs(T, H, Hkv, d, "f32", 3)
    rope = binding.Rope.of(32, 10000.0, interleaved)
    pos = torch.tensor([0, 1, 5, 100, 4000, 90000], dtype=torch.int32, device="cuda")
    dq, dk = (torch.randn(x.shape, generator=g).cuda() for x in (q, k))
    gq, gk, gwq, gwk = binding.qk_norm_rotate_backward(dq, dk, q, k, pos, rope, wq, wk)

    def loss(q, k, wq, wk):
        a, b = binding.qk_norm_rotate(q, k, pos, rope, wq, wk)
        return float((a.double() * dq.double()).sum() + (b.double() * dk.double()).sum())

    xs, gs, h = [q, k, wq, wk], [gq, gk, gwq, gwk], 2.0 ** -7
    for n in range(4):
        u = torch.randn(xs[n].shape, generator=g).cuda()
        up, down = list(xs), list(xs)
        up[n], down[n] = xs[n] + h * u, xs[n] - h * u
        slope, formula = (loss(*up) - loss(*down)) / (2 * h), float((gs[n].double() * u.double()).sum())
        size = float((gs[n].double().abs() * u.double().abs()).sum())
        assert abs(slope - formula) <= 1e-3 * size, (n, slope, formula, size)


def test_the_same_bits_every_time():
    q, k, (wq, wk), g = _inputs(5000, 8, 2, 64, "bf16", 8)
    rope = binding.Rope.of(64)
    dq, dk = (torch.randn(x.shape, generator=g).to(x.dtype).cuda() for x in (q, k))
    first = binding.qk_norm_rotate_backward(dq, dk, q, k, None, rope, wq, wk)
    for _ in range(3):
        again = binding.qk_norm_rotate_backward(dq, dk, q, k, None, rope, wq, wk)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


# ---------------------------------------------------------------- into pages
def _pool(io, d, Hkv, page, rows, seed, layers=1, spare=3, seqs=None):
    """An empty pool whose pages hold NaN, and sequences of rows[i] tokens in pages of random numbers."""
    seqs = len(rows) if seqs is None else seqs
    M = max(1, max(-(-n // page) for n in rows)) + 1
    P = sum(-(-n // page) for n in rows) + spare
    pool = binding.KvPages.empty(layers, P, Hkv, d, page, seqs, M, DT[io])
    pool.k_pages.fill_(float("nan"))
    pool.v_pages.fill_(float("nan"))
    order = torch.randperm(P, generator=torch.Generator().manual_seed(seed)).int()
    at = 0
    table, refs = pool.table.cpu(), pool.refs.cpu()
    for s, n in enumerate(rows):
        m = -(-n // page)
        table[s, :m] = order[at:at + m]
        refs[order[at:at + m].long()] = 1
        at += m
    pool.table.copy_(table)
    pool.refs.copy_(refs)
    pool.lens[:len(rows)].copy_(torch.tensor(rows, dtype=torch.int32))
    return pool


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("d,H,Hkv", [(64, 4, 2), (128, 3, 1)])
def test_append(io, page, d, H, Hkv):
    print(f"case page={page} d={d} {io}", flush=True)
    news, lens = [1, 0, 23, 8, 5, 70, 16], [1, 9, 40, 8, 333, 300, 32]
    B, layers, layer = len(news), 3, 1
    pool = _pool(io, d, Hkv, page, lens, page + d, layers)
    seqs = torch.tensor([3, 0, 5, 1, 6, 2, 4], dtype=torch.int32)
    n_of = [news[s] for s in seqs.tolist()]
    start = torch.tensor([0] + n_of).cumsum(0).int()
    T = int(start[-1])
    q, k, (wq, wk), g = _inputs(T, H, Hkv, d, io, 77, fused=True)
    v = torch.randn(T, Hkv, d, generator=g).to(DT[io]).cuda()
    v[3, 0, :5] = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0, -0.0])          # values are copied, whatever they are
    rope = binding.Rope.of(d, 500000.0)
    before = [x.cpu().clone() for x in (pool.k_pages, pool.v_pages)]
    out = pool.append(layer, q, k, v, start.cuda(), seqs.cuda(), rope, wq, wk)
    freq, table = ref.f64(rope.inv_freq), pool.table.cpu()
    kp, vp = pool.k_pages.cpu(), pool.v_pages.cpu()
    written = torch.zeros(pool.pages, page, dtype=torch.bool)
    for b, s in enumerate(seqs.tolist()):
        lo, hi = int(start[b]), int(start[b + 1])
        if lo == hi:
            continue
        pos = np.arange(lens[s] - (hi - lo), lens[s])
        for x, w, is_key in ((q, wq, False), (k, wk, True)):
            x64, w64 = ref.f64(x[lo:hi]), ref.f64(w)
            plain = ref.heads(x64, w64, pos, np.zeros(0), 1e-6)
            rows, vals = ref.pool_rows(kp, vp, layer, table[s, :-(-lens[s] // page)].long())
            y = rows[pos] if is_key else out[lo:hi]
            _check(y, ref.heads(x64, w64, pos, freq, 1e-6), _turn_size(plain, d // 2, False), DT[io], d)
        assert torch.equal(vals[pos].view(torch.int16 if io == "bf16" else torch.int32), v[lo:hi].cpu().contiguous().view(torch.int16 if io == "bf16" else torch.int32))
        for p in pos:
            written[int(table[s, p // page]), p % page] = True
    # every other token of every page and layer holds what it held
    bits = torch.int16 if io == "bf16" else torch.int32
    for now, was, groups in ((kp, before[0], False), (vp, before[1], True)):
        for L in range(layers):
            a, b = now[L].view(bits), was[L].view(bits)
            a, b = (x.permute(0, 2, 4, 1, 3).reshape(pool.pages, page, -1) if groups else x.permute(0, 3, 1, 2, 4).reshape(pool.pages, page, -1) for x in (a, b))
            same = (a == b).all(-1)
            assert (same | (written if L == layer else torch.zeros_like(written))).all()


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 130, 4200])
def test_append_of_many_sequences_is_that_of_each(B):
    """Which sequence a token is of is found among all of them; sequences without a new token in between, at the front and at the end."""
    print(f"case B={B}", flush=True)
    g = torch.Generator().manual_seed(B)
    news = torch.randint(0, 4, (B,), generator=g)
    news[B // 3] = 19
    news[0], news[-1] = (0, 0) if B > 2 else (3, 5)
    lens = (news + torch.randint(0, 13, (B,), generator=g)).tolist()
    pools = [_pool("bf16", 64, 1, 16, lens, 3) for _ in range(2)]
    start = torch.tensor([0] + news.tolist()).cumsum(0).int()
    T = int(start[-1])
    q, k, (wq, wk), _ = _inputs(T, 2, 1, 64, "bf16", 8)
    v, rope = k.flip(0).contiguous(), binding.Rope.of(64)
    out = pools[0].append(0, q, k, v, start.cuda(), None, rope, wq, wk)
    rows = torch.arange(B, dtype=torch.int32).cuda()
    for b in range(B):
        lo, hi = int(start[b]), int(start[b + 1])
        if hi > lo:
            one = torch.tensor([0, hi - lo], dtype=torch.int32).cuda()
            got = pools[1].append(0, q[lo:hi], k[lo:hi], v[lo:hi], one, rows[b:b + 1], rope, wq, wk)
            assert torch.equal(got, out[lo:hi]), b
    for x, y in ((pools[0].k_pages, pools[1].k_pages), (pools[0].v_pages, pools[1].v_pages)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_append_leaves_out_what_has_no_place():
    """Rows outside the table, sequences shorter than their new tokens, page numbers outside the pool: nothing is written anywhere."""
    pool = _pool("bf16", 64, 1, 16, [40, 3, 20], 1)
    pool.table[2, 1] = pool.pages + 7
    pool.table[0, 2] = -5
    before = pool.k_pages.clone(), pool.v_pages.clone()
    q, k, (wq, wk), g = _inputs(4 + 5 + 2 + 3, 2, 1, 64, "bf16", 4)
    v = k.clone()
    start = torch.tensor([0, 4, 9, 11, 14], dtype=torch.int32, device="cuda")
    pool4 = binding.KvPages(pool.k_pages, pool.v_pages, pool.book, 3, pool.max_pages)
    with pytest.raises(binding.SpectreError):
        pool4.append(0, q, k, v, start, None, None)                        # four sequences, three rows
    start = torch.tensor([0, 4, 9, 11], dtype=torch.int32, device="cuda")
    for seqs in ([0, 1, 2], [-1, 1, 3]):
        pool.append(0, q[:11], k[:11], v[:11], start, torch.tensor(seqs, dtype=torch.int32, device="cuda"), binding.Rope.of(64), wq, wk)
    bits = torch.int16
    assert torch.equal(pool.k_pages.view(bits), before[0].view(bits)) and torch.equal(pool.v_pages.view(bits), before[1].view(bits))
