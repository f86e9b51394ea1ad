"""The weights of few rows in bf16: two terms each, so that outputs are off by their own rounding and no more."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from test_gpu_attend import make, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,H,Hkv", [(64, 4, 1), (128, 2, 2), (64, 7, 1)])
@pytest.mark.parametrize("news,lens", [([1] * 8, [2, 3, 5, 17, 40, 129, 700, 4000]), ([2, 1, 2], [9, 300, 2500])])
@pytest.mark.parametrize("window", [0, 30])
def test_outputs_are_as_close_as_their_rounding(d, H, Hkv, news, lens, window):
    """A weight's first term leaves a rest of at most half a step of it, whose own rounding is half a step of that: u^2.  Values that cancel each other leave outputs far
    below the weights' sum, where one rounding of each weight would show."""
    print(f"case d={d} H={H} {news} window={window}", flush=True)
    pool, rows = make("bf16", d, Hkv, 16, lens, d + H)
    q, start = queries(news, H, d, "bf16", 8)
    out = pool.attend(0, q, start, max_new=max(news), max_len=max(lens), window=window)
    u, u32, at = ref.half_step(torch.bfloat16), 2.0 ** -24, 0
    for b, n in enumerate(news):
        k, v = rows[b]
        x = ref.f64(q[at:at + n])
        want, _ = ref.attend(x, k, v, d ** -0.5, window)
        size, _ = ref.attend(x, k, np.abs(v), d ** -0.5, window)
        score = d ** -0.5 * np.abs(x).max() * np.abs(k).max() * d * (d + 4) * u32
        tol = u * np.abs(want) + size * (1 + u) * (u * u + 2 * score + (len(k) + 24) * u32)
        err = np.abs(ref.f64(out[at:at + n]) - want)
        assert (err <= tol).all(), f"sequence {b}: {float((err / tol).max())} of the bound"
        at += n


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 3])
def test_values_that_are_not_finite_among_many(io, d, n):
    """Infinities and NaN far from the ends of a sequence reach the channel that they are in, of every row, and no other one."""
    print(f"case {io} d={d} n={n}", flush=True)
    m, H = 3000, 4
    pool, rows = make(io, d, 1, 64, [m], n + d)
    E, table, k, v = ref.per_group(pool.dtype), pool.table.cpu(), *rows[0]
    bad = {3: float("inf"), 17: -float("inf"), d - 1: float("nan")}
    for at, (ch, x) in zip((11, 1500, 2222), bad.items()):
        pool.v_pages[0, int(table[0, at // 64]), 0, at % 64 // E, ch, at % E] = x
        v[at, 0, ch] = 0.0                                       # stands for it where the other channels are compared
    q, start = queries([n], H, d, io, 3)
    out, lse = pool.attend(0, q, start, max_new=n, max_len=m, want_lse=True)
    got = ref.f64(out)
    assert (got[..., 3] == np.inf).all() and (got[..., 17] == -np.inf).all() and np.isnan(got[..., d - 1]).all() and torch.isfinite(lse).all()
    want, _ = ref.attend(ref.f64(q), k, v, d ** -0.5)
    tol = ref.attend_bound(ref.f64(q), k, v, d ** -0.5, pool.dtype)
    rest = [c for c in range(d) if c not in bad]
    assert (np.abs(got - want) <= tol)[..., rest].all()
