"""Norm and rotation of heads by positions of several axes on the GPU against the 64-bit form: values, gradients, pages."""
import numpy as np
import pytest
import torch

import axes_ref
import paged_ref as ref
from paper_2502_18394_amd import binding
from test_gpu_heads import DT, U32, _check, _inputs, _turn_size

pytestmark = pytest.mark.gpu

CASES = [  # T, H, Hkv, d, rot, axes, interleaved, norm
    (1, 1, 1, 64, 64, 3, False, True), (7, 5, 5, 64, 64, 2, True, True), (8, 4, 2, 128, 128, 3, False, True), (9, 3, 1, 128, 32, 4, False, True),
    (17, 7, 7, 64, 16, 8, True, True), (33, 6, 2, 128, 128, 3, True, False), (1003, 32, 8, 64, 64, 3, False, True), (0, 4, 2, 64, 64, 3, False, True),
]


def _rope(rot, axes, interleaved, g):
    """Every axis has a pair; the others go to any."""
    axis = torch.cat((torch.arange(axes), torch.randint(0, axes, (rot // 2 - axes,), generator=g)))[torch.randperm(rot // 2, generator=g)]
    return binding.Rope.of(rot, 500000.0, interleaved, axes=axis), axis.numpy()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,Hkv,d,rot,axes,interleaved,norm", CASES)
def test_forward_and_backward(T, H, Hkv, d, rot, axes, interleaved, norm, io):
    print(f"case T={T} H={H} Hkv={Hkv} d={d} rot={rot} axes={axes} {io}", flush=True)
    q, k, w, g = _inputs(T, H, Hkv, d, io, T + d + rot, fused=T == 33)
    rope, axis = _rope(rot, axes, interleaved, g)
    pos = torch.randint(-1000, 1 << 20, (axes, T), generator=g, dtype=torch.int32)
    if T > 2:
        pos[0, 0], pos[1, 1], pos[-1, 2] = 0, 2 ** 31 - 1, -2 ** 31
    angle = axes_ref.angles(pos, axis, ref.f64(rope.inv_freq))
    wq, wk = w if norm else (None, None)
    got = binding.qk_norm_rotate(q, k, pos.cuda(), rope, wq, wk, 1e-5)
    dy = [torch.randn(x.shape, generator=g).to(DT[io]).cuda() for x in (q, k)]
    grads = binding.qk_norm_rotate_backward(*dy, q, k, pos.cuda(), rope, wq, wk, 1e-5)
    for n, (x, weight) in enumerate(((q, wq), (k, wk))):
        x64, w64 = ref.f64(x), None if weight is None else ref.f64(weight)
        plain = axes_ref.heads(x64, w64, angle * 0, 1e-5, interleaved)
        _check(got[n], axes_ref.heads(x64, w64, angle, 1e-5, interleaved), _turn_size(plain, rot // 2, interleaved), DT[io], d)
        d64 = ref.f64(dy[n])
        want, want_w = axes_ref.heads_backward(d64, x64, w64, angle, 1e-5, interleaved)
        size = _turn_size(d64, rot // 2, interleaved)
        if not norm:
            _check(grads[n], want, size, DT[io], d)
            continue
        r = 1 / np.sqrt((x64 * x64).mean(-1, keepdims=True) + 1e-5)
        h, xh = size * np.abs(w64), np.abs(x64 * r)
        _check(grads[n], want, 3 * r * (h + xh * (h * xh).mean(-1, keepdims=True)), DT[io], d)
        # products and the sums of one run of 8 tokens in 32 bits (at most 8 H terms), the rest in 64, one rounding
        tol = (d + 16 + 8 * H) * U32 * (size * xh).sum((0, 1)) + U32 * np.abs(want_w) + 1e-300
        assert (np.abs(ref.f64(grads[2 + n]) - want_w) <= tol).all()


def test_gradients_against_differences():
    """The slope of sum(dy * y) along a direction, from the GPU's fp32 forward pass at x +- h u, as for one axis: off by h^2 / 6 of the third derivative (below 1e-4
    of the slope's size) and by rounding, 2 * 2^-24 sqrt(terms) |dy y| / h."""
    q, k, (wq, wk), g = _inputs(6, 3, 2, 64, "f32", 3)
    rope, _ = _rope(48, 3, False, g)
    pos = torch.randint(0, 90000, (3, 6), generator=g, dtype=torch.int32).cuda()
    dq, dk = (torch.randn(x.shape, generator=g).cuda() for x in (q, k))
    gs = binding.qk_norm_rotate_backward(dq, dk, q, k, pos, rope, wq, wk)

    def loss(*xs):
        a, b = binding.qk_norm_rotate(xs[0], xs[1], pos, rope, xs[2], xs[3])
        return float((a.double() * dq.double()).sum() + (b.double() * dk.double()).sum())

    xs, h = [q, k, wq, wk], 2.0 ** -7
    for n in range(4):
        u = torch.randn(xs[n].shape, generator=g).cuda()
        up, down = list(xs), list(xs)
        up[n], down[n] = xs[n] + h * u, xs[n] - h * u
        slope, formula = (loss(*up) - loss(*down)) / (2 * h), float((gs[n].double() * u.double()).sum())
        assert abs(slope - formula) <= 1e-3 * float((gs[n].double().abs() * u.double().abs()).sum()), n


def test_axes_that_agree_are_one_axis():
    q, k, (wq, wk), g = _inputs(77, 4, 2, 64, "bf16", 9)
    pos = torch.randint(0, 100000, (77,), generator=g, dtype=torch.int32).cuda()
    rope, _ = _rope(64, 3, False, g)
    a = binding.qk_norm_rotate(q, k, pos.expand(3, 77).contiguous(), rope, wq, wk)
    b = binding.qk_norm_rotate(q, k, pos, binding.Rope.of(64, 500000.0), wq, wk)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("page,d", [(16, 64), (64, 128)])
def test_append_at_positions(io, page, d):
    """Rotated by the positions given, stored by the order of the tokens; what is not the new tokens' stays as it was."""
    print(f"case {io} page={page} d={d}", flush=True)
    H, Hkv, news, had, seqs = 6, 2, [5, 0, 1, 40], [9, 3, 0, 61], [2, 0, 3, 1]
    T, g = sum(news), torch.Generator().manual_seed(page)
    pool = binding.KvPages.empty(2, 40, Hkv, d, page, 5, 12, DT[io])
    rows = torch.tensor(seqs, dtype=torch.int32, device="cuda")
    pool.reserve(rows, torch.tensor([a + b for a, b in zip(news, had)], dtype=torch.int32, device="cuda"))
    for x in (pool.k_pages, pool.v_pages):
        x.copy_(torch.randn(x.shape, generator=g).to(x.dtype))
    before = pool.k_pages.cpu().clone(), pool.v_pages.cpu().clone()
    q, k, v = (torch.randn(T, n, d, generator=g).to(DT[io]).cuda() for n in (H, Hkv, Hkv))
    rope, axis = _rope(d, 3, False, g)
    pos = torch.randint(0, 90000, (3, T), generator=g, dtype=torch.int32)
    start = torch.tensor([0] + news).cumsum(0).int()
    w = [(1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in "qk"]
    out = pool.append(1, q, k, v, start.cuda(), rows, rope, *w, positions=pos.cuda())
    both = binding.qk_norm_rotate(q, k, pos.cuda(), rope, *w)
    assert torch.equal(out, both[0])
    table = pool.table.cpu()
    want = [x.clone() for x in before]
    E = ref.per_group(DT[io])
    for b, n in enumerate(news):
        for i in range(n):
            t, at = int(start[b]) + i, had[b] + i
            number, slot = int(table[seqs[b], at // page]), at % page
            want[0][1, number, :, :, slot] = both[1][t].cpu().view(Hkv, d // E, E)
            want[1][1, number, :, slot // E, :, slot % E] = v[t].cpu()
    assert torch.equal(pool.k_pages.cpu(), want[0]) and torch.equal(pool.v_pages.cpu(), want[1]) and int(pool.status[0]) == 0
    # without axes: positions of one axis given are the same as found, where they are the places
    one = binding.Rope.of(d)
    places = torch.cat([torch.arange(a, a + n) for n, a in zip(news, had)]).int().cuda()
    a = pool.append(0, q, k, v, start.cuda(), rows, one, *w, positions=places)
    pages = pool.k_pages[0].clone()
    b = pool.append(0, q, k, v, start.cuda(), rows, one, *w)
    assert torch.equal(a, b) and torch.equal(pages, pool.k_pages[0])


def test_captured_with_new_positions():
    """A graph of forward and backward, replayed with positions and rows that changed, with eager work between the replays."""
    q, k, (wq, wk), g = _inputs(50, 4, 2, 64, "bf16", 4)
    rope, _ = _rope(64, 3, True, g)
    pos = torch.zeros(3, 50, dtype=torch.int32, device="cuda")
    dq, dk = q.clone(), k.clone()
    step = lambda: binding.qk_norm_rotate(q, k, pos, rope, wq, wk) + binding.qk_norm_rotate_backward(dq, dk, q, k, pos, rope, wq, wk)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(3):
        pos.copy_(torch.randint(0, 70000, pos.shape, generator=g, dtype=torch.int32))
        for x in (q, k, dq, dk):
            x.copy_(torch.randn(x.shape, generator=g))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
