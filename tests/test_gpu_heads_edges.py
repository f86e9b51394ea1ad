"""Norm and rotation of heads where sums, padding rows and untouched channels can go wrong."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2502_18394_amd import binding
from test_gpu_heads import DT, U32, _check, _inputs, _pool, _turn_size

pytestmark = pytest.mark.gpu
CHAIN = 128                                          # rows that a thread adds in 32 bits before they go into 64, at most


def _weights_close(got, want, terms, d):
    """A product of three roundings around a sum of d squares, sums of up to CHAIN products in 32 bits, the rest in 64, one rounding."""
    tol = (d + 16 + CHAIN) * U32 * terms + U32 * np.abs(want) + 1e-300
    err = np.abs(ref.f64(got) - want)
    assert np.isfinite(ref.f64(got)).all() and (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,Hkv,d", [(1, 1, 1, 64), (1, 3, 2, 128), (7, 4, 1, 64), (9, 5, 5, 64), (9, 2, 1, 128), (16, 3, 4, 64)])
def test_no_epsilon(T, H, Hkv, d, io):
    """eps = 0 is a norm like any other while no row is all zero: what pads a workgroup's tokens and heads is no row."""
    print(f"case T={T} H={H} Hkv={Hkv} d={d} {io}", flush=True)
    q, k, w, g = _inputs(T, H, Hkv, d, io, T + H + d)
    dy = [torch.randn(x.shape, generator=g).to(DT[io]).cuda() for x in (q, k)]
    rope, pos = binding.Rope.of(d), np.arange(T)
    freq = ref.f64(rope.inv_freq)
    got = binding.qk_norm_rotate(q, k, None, rope, *w, 0.0)
    grads = binding.qk_norm_rotate_backward(*dy, q, k, None, rope, *w, 0.0)
    for n, (x, weight) in enumerate(((q, w[0]), (k, w[1]))):
        x64, w64, d64 = ref.f64(x), ref.f64(weight), ref.f64(dy[n])
        _check(got[n], ref.heads(x64, w64, pos, freq, 0.0), _turn_size(ref.heads(x64, w64, pos, np.zeros(0), 0.0), d // 2, False), DT[io], d)
        want, want_w = ref.heads_backward(d64, x64, w64, pos, freq, 0.0)
        size = _turn_size(d64, d // 2, False)
        r = 1 / np.sqrt((x64 * x64).mean(-1, keepdims=True))
        h, xh = size * np.abs(w64), np.abs(x64 * r)
        _check(grads[n], want, 3 * r * (h + xh * (h * xh).mean(-1, keepdims=True)), DT[io], d)
        _weights_close(grads[2 + n], want_w, (size * xh).sum((0, 1)), d)


@pytest.mark.parametrize("T,H,Hkv", [(1, 65536, 1), (1, 1, 40000), (17, 5000, 300)])
def test_weight_gradients_of_very_many_heads(T, H, Hkv):
    """Heads that are all alike: a long sum of equal terms in 32 bits is off by much more than its terms are."""
    print(f"case T={T} H={H} Hkv={Hkv}", flush=True)
    d = 64
    q, k, w, g = _inputs(T, 1, 1, d, "f32", 4)
    dq, dk = (torch.randn(T, 1, d, generator=g).cuda() for _ in "qk")
    many = lambda x, n: x.expand(T, n, d).contiguous()
    grads = binding.qk_norm_rotate_backward(many(dq, H), many(dk, Hkv), many(q, H), many(k, Hkv), None, None, *w, 1e-6)
    for n, (x, dy, heads) in enumerate(((q, dq, H), (k, dk, Hkv))):
        _, want = ref.heads_backward(ref.f64(dy), ref.f64(x), ref.f64(w[n]), np.zeros(T), np.zeros(0), 1e-6)
        x64 = ref.f64(x)
        xh = np.abs(x64 / np.sqrt((x64 * x64).mean(-1, keepdims=True) + 1e-6))
        _weights_close(grads[2 + n], heads * want, heads * (np.abs(ref.f64(dy)) * xh).sum((0, 1)), d)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,Hkv,d", [(9001, 2, 1, 64), (33003, 1, 1, 64), (25001, 3, 1, 128)])
def test_backward_of_several_runs_a_workgroup(T, H, Hkv, d, io):
    """So many tokens that a workgroup has more than one run of them, whole and ragged ones."""
    print(f"case T={T} H={H} Hkv={Hkv} d={d} {io}", flush=True)
    q, k, w, g = _inputs(T, H, Hkv, d, io, T)
    dy = [torch.randn(x.shape, generator=g).to(DT[io]).cuda() for x in (q, k)]
    rope, pos = binding.Rope.of(d, 500000.0), np.arange(T)
    freq = ref.f64(rope.inv_freq)
    grads = binding.qk_norm_rotate_backward(*dy, q, k, None, rope, *w, 1e-5)
    for n, (x, weight) in enumerate(((q, w[0]), (k, w[1]))):
        x64, w64, d64 = ref.f64(x), ref.f64(weight), ref.f64(dy[n])
        want, want_w = ref.heads_backward(d64, x64, w64, pos, freq, 1e-5)
        size = _turn_size(d64, d // 2, False)
        r = 1 / np.sqrt((x64 * x64).mean(-1, keepdims=True) + 1e-5)
        h, xh = size * np.abs(w64), np.abs(x64 * r)
        _check(grads[n], want, 3 * r * (h + xh * (h * xh).mean(-1, keepdims=True)), DT[io], d)
        _weights_close(grads[2 + n], want_w, (size * xh).sum((0, 1)), d)


def _same_bits(a, b):
    bits = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 16), (64, 48), (128, 32)])
def test_channels_that_are_not_turned_pass_through(d, rot, interleaved, io):
    """Without a norm they are copies, whatever they hold, and nothing of theirs reaches another channel: forward, backward and into pages."""
    print(f"case d={d} rot={rot} interleaved={interleaved} {io}", flush=True)
    T, H, Hkv = 11, 4, 2
    q, k, _, _ = _inputs(T, H, Hkv, d, io, rot)
    odd = [x.clone() for x in (q, k)]
    for x in odd:
        x[:, :, rot + 1] = float("inf")
        x[::2, :, rot + 4] = float("nan")
        x[1::2, :, d - 1] = -float("inf")
        x[:, :, rot + 2] = -0.0
    rope = binding.Rope.of(rot, 10000.0, interleaved)
    pos = torch.arange(5, 5 + T, dtype=torch.int32, device="cuda")
    for call in (lambda q, k: binding.qk_norm_rotate(q, k, pos, rope), lambda q, k: binding.qk_norm_rotate_backward(q, k, q, k, pos, rope)[:2]):
        for got, plain, x in zip(call(*odd), call(q, k), odd):
            assert _same_bits(got[..., rot:], x[..., rot:])
            assert _same_bits(got[..., :rot], plain[..., :rot])
    pool = _pool(io, d, Hkv, 16, [T], 1)
    start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    out = pool.append(0, odd[0], odd[1], odd[1], start, None, rope)
    keys, _ = ref.pool_rows(pool.k_pages.cpu(), pool.v_pages.cpu(), 0, pool.table[0, :1].cpu().long())
    assert _same_bits(out[..., rot:], odd[0][..., rot:]) and _same_bits(keys[:T, :, rot:], odd[1][..., rot:].cpu())
    assert torch.isfinite(out[..., :rot]).all() and torch.isfinite(keys[:T, :, :rot]).all()
