"""Residual and norm: what is refused on the host before anything is launched (no device is touched), and the 64-bit form the GPU tests rest on."""
import os

import numpy as np
import pytest
import torch

import norm_ref as ref
from paper_2502_18394_amd import binding

FAKE, FAR, OUT, BIG = 1 << 20, 1 << 40, 1 << 41, 1 << 30        # never dereferenced: every call below fails its checks first
W, SCALES = 1 << 24, 1 << 42


@pytest.fixture(scope="module")
def lib():
    from paper_2502_18394_amd import build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


def test_forward_refuses(lib):
    def forward(x=FAKE, xs=256, delta=FAR, ds=256, w=W, T=3, D=256, eps=1e-6, io=1, total=OUT, y=OUT + BIG, kind=1, scales=None):
        return lib.spectre_norm_forward(x, xs, delta, ds, w, T, D, eps, io, total, y, kind, scales, None)

    for bad, code in ((dict(x=None), 1), (dict(x=FAKE + 8), 1), (dict(xs=255), 1), (dict(xs=260), 1), (dict(delta=None), 1), (dict(total=None), 1), (dict(ds=128), 1),
                      (dict(w=W + 4), 1), (dict(T=-1), 1), (dict(D=0), 1), (dict(D=250), 2), (dict(D=1 << 15, xs=1 << 15, ds=1 << 15), 2), (dict(eps=-1.0), 1),
                      (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(io=4), 1), (dict(io=2), 1), (dict(y=None), 1), (dict(y=OUT + BIG + 8), 1),
                      (dict(kind=0), 1), (dict(kind=4), 1), (dict(scales=SCALES), 1), (dict(kind=4, scales=SCALES, D=192), 2), (dict(y=FAKE), 1), (dict(y=FAR + 512), 1),
                      (dict(total=FAKE), 1), (dict(y=OUT + 16), 1), (dict(kind=4, scales=OUT + 16), 1), (dict(kind=4, scales=SCALES + 2), 1),
                      (dict(io=0, kind=0, D=8196, xs=8196, ds=8196), 2)):
        assert forward(**bad) == code, bad
        assert lib.spectre_last_error()
    assert forward(T=0, x=None, y=None) == 0


def test_backward_refuses(lib):
    need = lib.spectre_norm_backward_workspace_bytes(3000, 256, 1)
    assert need >= 3000 // 128 * 256 * 4 and lib.spectre_norm_backward_workspace_bytes(3, 256, 1) == 0       # one workgroup's sums are the gradient
    assert lib.spectre_norm_backward_workspace_bytes(3000, 250, 1) == 0 and lib.spectre_norm_backward_workspace_bytes(3000, 256, 4) == 0
    assert lib.spectre_norm_backward_workspace_bytes(-1, 256, 1) == 0
    # the sums of 32 bits are of 128 rows at most: so many rows of partial sums
    assert lib.spectre_norm_backward_workspace_bytes(10 ** 7, 64, 1) >= 10 ** 7 // 128 * 64 * 4

    def backward(dy=FAKE, ys=256, total=FAR, ts=256, dsum=FAR + BIG, ds=256, w=W, T=3000, D=256, eps=1e-6, io=1, gx=OUT, gw=OUT + BIG, ws=W + BIG, size=need):
        return lib.spectre_norm_backward(dy, ys, total, ts, dsum, ds, w, T, D, eps, io, gx, gw, ws, size, None)

    for bad, code in ((dict(dy=None), 1), (dict(total=None), 1), (dict(dsum=FAR + BIG + 4), 1), (dict(ds=128), 1), (dict(gx=None), 1), (dict(gx=FAR), 1), (dict(gx=FAKE), 1),
                      (dict(gx=FAR + BIG), 1), (dict(gw=OUT + 16), 1), (dict(gw=FAKE), 1), (dict(ws=None), 3), (dict(size=need - 256), 3), (dict(ws=W + BIG + 4), 1),
                      (dict(D=200), 1), (dict(D=4), 2), (dict(io=3), 1), (dict(eps=-0.5), 1), (dict(gw=OUT + BIG + 2), 1), (dict(gw=OUT + BIG + 4), 1)):
        a = dict(bad)
        if a.get("D") == 200:
            a["ys"] = 199
        assert backward(**a) == code, bad
    assert backward(T=0, gw=None, dy=None) == 0


def test_the_binding_refuses():
    x = torch.zeros(3, 256, dtype=torch.bfloat16)
    for bad, error in ((dict(x=x), ValueError), (dict(x=x.half()), TypeError), (dict(x=x, dtype=torch.float32), TypeError), (dict(x=x, dtype=torch.float8_e5m2), TypeError)):
        with pytest.raises(error):
            binding.add_norm(**bad)
    with pytest.raises(ValueError):
        binding.add_norm_backward(x, x)


@pytest.mark.parametrize("weight,residual", [(True, True), (False, True), (True, False)])
def test_gradient_formula_against_differences(weight, residual):
    r = np.random.default_rng(4)
    s, w, dy, e = r.normal(size=(3, 12)), r.normal(size=12) if weight else None, r.normal(size=(3, 12)), r.normal(size=(3, 12)) if residual else None
    gx, gw = ref.norm_backward(dy, s, w, e, 1e-3)
    loss = lambda s, w: (ref.norm(s, w, 1e-3) * dy).sum() + (0 if e is None else (s * e).sum())
    h = 1e-6
    for i in np.ndindex(s.shape):
        d = np.zeros_like(s)
        d[i] = h
        assert abs((loss(s + d, w) - loss(s - d, w)) / (2 * h) - gx[i]) < 1e-7
    if weight:
        for i in range(12):
            d = np.zeros(12)
            d[i] = h
            assert abs((loss(s, w + d) - loss(s, w - d)) / (2 * h) - gw[i]) < 1e-7
