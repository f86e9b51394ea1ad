"""A residual's addition and the norm of the sum on the GPU against the 64-bit form: values, gradients, rows in 8 bits."""
import numpy as np
import pytest
import torch

import e4m3_ref
import norm_ref as ref
import paged_ref
from paper_2502_18394_amd import binding

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U32 = 2.0 ** -24
f64 = paged_ref.f64

# T, D: one row, as many as a workgroup has and one more, a row that ends inside every size of a workgroup
SHAPES = [(1, 8), (3, 16), (5, 504), (4, 512), (9, 520), (2, 1024), (7, 1032), (1, 2048), (33, 2056), (6, 4096), (3, 4104), (5, 8192), (2, 7992), (1000, 128), (3001, 256), (0, 64)]


def _inputs(T, D, io, seed, strided=False, scale=3.0):
    g = torch.Generator().manual_seed(seed)
    wide = 16 if strided else 0                              # something between the rows
    r = lambda s: (torch.randn(T, D + wide, generator=g) * s).to(DT[io]).cuda()[:, :D]
    return r(scale), r(1.0), (1 + 0.2 * torch.randn(D, generator=g)).cuda(), g


def _sum(x, delta, dtype):
    """What is kept of the sum: one rounding of the sum of two numbers, which torch's addition is, too."""
    return x + delta if delta is not None else x


def _check_norm(y, s, w, eps, dtype, D):
    """One rounding to the type, and 32-bit arithmetic: a sum of D squares (a bound; what it really is grows with the root), a root, three products."""
    want = ref.norm(f64(s), w, eps)
    assert (np.abs(f64(y) - want) <= paged_ref.half_step(dtype) * np.abs(want) + (D + 16) * U32 * np.abs(want) + 1e-37).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T,D", SHAPES + [(3, 16384)])
def test_forward(T, D, io):
    print(f"case T={T} D={D} {io}", flush=True)
    if io == "f32" and D > 8192:
        with pytest.raises(binding.SpectreError):
            binding.add_norm(torch.zeros(T, D, device="cuda"))
        return
    for strided in (False, True):
        x, delta, w, _ = _inputs(T, D, io, T + D, strided)
        total, y = binding.add_norm(x, w, delta, 1e-5)
        assert total.dtype == y.dtype == x.dtype and torch.equal(total, x + delta)
        _check_norm(y, total, f64(w), 1e-5, DT[io], D)
        same, y = binding.add_norm(x, w, eps=1e-5)
        assert same is x
        _check_norm(y, x, f64(w), 1e-5, DT[io], D)
        _, y = binding.add_norm(x, None, delta, 0.0)
        _check_norm(y, x + delta, None, 0.0, DT[io], D)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T,D", [(1, 128), (5, 256), (3, 1152), (2, 2048), (7, 4096), (3, 8192), (1001, 384), (0, 128)])
def test_rows_in_8_bits(T, D, io):
    print(f"case T={T} D={D} {io}", flush=True)
    x, delta, w, _ = _inputs(T, D, io, T + D, strided=T == 7)
    if T > 2:
        x[1], delta[1] = 0, 0                                # a row of nothing
        x[2, 128:256] = 0
        if D > 128:
            delta[2, 128:256] = 0
    total, codes, scales = binding.add_norm(x, w, delta, 1e-5, dtype=torch.float8_e4m3fn)
    assert torch.equal(total, x + delta) and codes.dtype == torch.float8_e4m3fn and tuple(scales.shape) == (T, D // 128)
    want = ref.norm(f64(total), f64(w), 1e-5)
    off = (D + 16) * U32                                     # relative, of the norm in 32 bits
    top = ref.scales(want)
    assert (np.abs(f64(scales) - top) <= (off + 4 * U32) * top).all()
    got = e4m3_ref.numbers(codes).numpy() * np.repeat(f64(scales), 128, 1)
    step = np.repeat(top, 128, 1)
    # one rounding to 8 bits, of a number that is off by the norm's arithmetic and by that of its scale
    assert (np.abs(got - want) <= e4m3_ref.STEP * np.abs(want) * (1 + 2 * off) + e4m3_ref.SMALL * step + (2 * off + 8 * U32) * np.abs(want)).all()
    if T > 2:
        assert (got[1] == 0).all() and (f64(scales)[1] == 0).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T,D", SHAPES + [(9000, 64), (8, 2048), (9, 2048), (32, 1024), (33, 1024), (8, 4096)])
def test_backward(T, D, io):
    print(f"case T={T} D={D} {io}", flush=True)
    s, dy, w, g = _inputs(T, D, io, T + D + 1, strided=T == 33)
    dsum = torch.randn(T, D, generator=g).to(DT[io]).cuda()
    for weight, e in ((w, dsum), (w, None), (None, dsum)):
        gx, gw = binding.add_norm_backward(dy, s, weight, e, 1e-5)
        w64, e64 = None if weight is None else f64(weight), None if e is None else f64(e)
        want, want_w = ref.norm_backward(f64(dy), f64(s), w64, e64, 1e-5)
        s64, h = f64(s), np.abs(f64(dy)) * (1 if weight is None else np.abs(w64))
        r = 1 / np.sqrt((s64 * s64).mean(-1, keepdims=True) + 1e-5)
        u = np.abs(s64 * r)
        size = 3 * r * (h + u * (h * u).mean(-1, keepdims=True)) + (0 if e is None else np.abs(e64))
        assert (np.abs(f64(gx) - want) <= paged_ref.half_step(DT[io]) * np.abs(want) + (D + 16) * U32 * size + 1e-37).all()
        if weight is None:
            assert gw is None
            continue
        # products, each off by the norm's root, sums of up to 128 of them in 32 bits, the others in 64, one rounding
        tol = (D + 16 + 128) * U32 * (np.abs(f64(dy)) * u).sum(0) + U32 * np.abs(want_w) + 1e-37
        assert (np.abs(f64(gw) - want_w) <= tol).all()


def test_gradients_against_differences():
    """The slope of sum(dy y) + sum(e s) along a direction, from the GPU's fp32 forward pass at +- h: off by h^2 / 6 of the third derivative (below 1e-4 of the slope's
    size) and by rounding, 2 * 2^-24 sqrt(terms) |dy y| / h."""
    x, dy, w, g = _inputs(7, 264, "f32", 6, scale=1.0)
    delta, e = (torch.randn(7, 264, generator=g).cuda() for _ in range(2))
    total, _ = binding.add_norm(x, w, delta)
    gx, gw = binding.add_norm_backward(dy, total, w, e)

    def loss(x, delta, w):
        s, y = binding.add_norm(x, w, delta)
        return float((y.double() * dy.double()).sum() + (s.double() * e.double()).sum())

    xs, gs, h = [x, delta, w], [gx, gx, gw], 2.0 ** -7
    for n in range(3):
        u = torch.randn(xs[n].shape, generator=g).cuda()
        up, down = list(xs), list(xs)
        up[n], down[n] = xs[n] + h * u, xs[n] - h * u
        slope, formula = (loss(*up) - loss(*down)) / (2 * h), float((gs[n].double() * u.double()).sum())
        assert abs(slope - formula) <= 1e-3 * float((gs[n].double().abs() * u.double().abs()).sum()), n


def test_not_finite_rows_stay_their_own():
    """NaN and infinities are their row's business: NaN throughout, or where the infinity stands; the other rows, and the backward pass of theirs, know nothing of them."""
    x, delta, w, _ = _inputs(6, 256, "bf16", 3)
    clean = binding.add_norm(x, w, delta)[1].clone()
    x[1, 7], x[3, 200], delta[4, 0] = float("nan"), float("inf"), float("-inf")
    _, y = binding.add_norm(x, w, delta)
    fine = [0, 2, 5]
    assert torch.equal(y[fine], clean[fine]) and y[1].isnan().all()
    bad = y.isnan()
    assert bad[3].sum() == 1 and bad[3, 200] and bad[4].sum() == 1 and bad[4, 0] and (y[3][~bad[3]] == 0).all()
    total, codes, scales = binding.add_norm(x, w, delta, dtype=torch.float8_e4m3fn)
    got = e4m3_ref.numbers(codes).numpy()
    assert np.isfinite(got[fine]).all() and np.isnan(got[1]).all() and torch.isnan(scales[1]).all() and torch.isfinite(scales[fine]).all()
    assert np.isnan(got[3, 128:]).any() and (got[3, :128] == 0).all()


def test_the_same_bits_every_time_and_on_another_stream():
    x, dy, w, g = _inputs(5000, 1024, "bf16", 2)
    first = binding.add_norm_backward(dy, x, w, dy)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    for where in (None, stream, None):
        again = binding.add_norm_backward(dy, x, w, dy, stream=where)
        forward = binding.add_norm(x, w, dy, stream=where)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again)) and torch.equal(forward[0], x + dy)


def test_outputs_that_are_given():
    x, delta, w, _ = _inputs(5, 256, "bf16", 1)
    total, y = torch.empty_like(x), torch.empty_like(x)
    got = binding.add_norm(x, w, delta, sum_out=total, out=y)
    assert got[0] is total and got[1] is y and torch.equal(total, x + delta)
    for bad in (dict(sum_out=x), dict(out=delta), dict(sum_out=y, out=y), dict(out=y[:4]), dict(out=y.float()), dict(scales=torch.empty(5, 2, device="cuda"))):
        with pytest.raises((ValueError, binding.SpectreError)):
            binding.add_norm(x, w, delta, **bad)
    with pytest.raises(ValueError):
        binding.add_norm(x[:, ::2], w)
    with pytest.raises(ValueError):
        binding.add_norm(x, w[:8])
    with pytest.raises(ValueError):
        binding.add_norm(x, w, delta[:4])


def test_captured():
    """Forward and backward in one graph, replayed on new rows with eager work between the replays."""
    x, delta, w, g = _inputs(300, 512, "bf16", 9)
    dy = x.clone()

    def step():
        total, y = binding.add_norm(x, w, delta)
        coded = binding.add_norm(x, w, delta, dtype=torch.float8_e4m3fn)
        return (total, y, coded[1].view(torch.uint8), coded[2]) + binding.add_norm_backward(dy, total, w, delta)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(3):
        for t in (x, delta, dy):
            t.copy_(torch.randn(t.shape, generator=g))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
