"""Positions of several axes: what is refused on the host before anything is launched (no device is touched), and the 64-bit form the GPU tests rest on."""
import ctypes
import os

import numpy as np
import pytest
import torch

import axes_ref as ref
import paged_ref
from paper_2502_18394_amd import binding

FAKE, FAR, OUT, BIG = 1 << 20, 1 << 40, 1 << 41, 1 << 30        # never dereferenced: every call below fails its checks first


@pytest.fixture(scope="module")
def lib():
    from paper_2502_18394_amd import build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


def heads(**change):
    P = dict(d=64, rot=64, interleaved=0, eps=1e-6, inv_freq=FAKE, wq=FAKE, wk=FAKE, axes=3, axis=FAKE)
    P.update(change)
    return ctypes.byref(binding.HeadsC(*P.values()))


@pytest.mark.parametrize("change,positions,code", [
    (dict(axes=-1), FAKE, 1), (dict(axes=9), FAKE, 2), (dict(axis=None), FAKE, 1), (dict(), None, 1), (dict(axis=FAKE + 2), FAKE, 1), (dict(), FAKE + 1, 1),
    (dict(axes=1, axis=None), FAKE + 2, 1)])
def test_axes_that_are_refused(lib, change, positions, code):
    P = heads(**change)
    kv = ctypes.byref(binding.KvC(2, 8, 2, 64, 16, 4, 5, binding.BF16, FAR, FAR + BIG, FAKE))
    assert lib.spectre_heads_forward(P, FAKE, 256, FAR, 128, positions, 3, 4, 2, 1, OUT, OUT + BIG, None) == code
    assert lib.spectre_heads_backward(P, FAKE, 256, FAR, 128, FAKE, 256, FAR, 128, positions, 3, 4, 2, 1, OUT, OUT + BIG, FAKE, FAKE, FAKE, BIG, None) == code
    assert lib.spectre_kv_append_at(kv, 0, P, FAKE, 256, FAR, 128, FAR, 128, positions, FAKE, None, 1, 3, 4, OUT, None) == code
    assert lib.spectre_last_error()


def test_append_without_positions_needs_one_axis(lib):
    kv = ctypes.byref(binding.KvC(2, 8, 2, 64, 16, 4, 5, binding.BF16, FAR, FAR + BIG, FAKE))
    assert lib.spectre_kv_append(kv, 0, heads(), FAKE, 256, FAR, 128, FAR, 128, FAKE, None, 1, 3, 4, OUT, None) == 1
    assert b"positions" in lib.spectre_last_error()
    # no token, no position
    assert lib.spectre_kv_append(kv, 0, heads(), None, 256, None, 128, None, 128, FAKE, None, 0, 0, 4, OUT, None) == 0


def test_ropes_that_are_refused():
    freq = torch.ones(4, dtype=torch.float64)
    for axes in ([0, 1, 2], [0, 1, 2, 8], [0, -1, 2, 3], [0.0, 1.0, 2.0, 0.0], [True, False, True, False], 1):
        with pytest.raises(ValueError):
            binding.Rope(freq, device="cpu", axes=axes)
    rope = binding.Rope(freq, device="cpu", axes=[0, 2, 2, 0])
    assert rope.axes == 3 and rope.axis.tolist() == [0, 2, 2, 0] and rope.axis.dtype == torch.int32
    assert binding.Rope(freq, device="cpu", axes=[0] * 4).axes == 1 and binding.Rope.of(64, device="cpu").axis is None
    for positions, error in ((None, ValueError), (torch.zeros(3, 5), TypeError), (torch.zeros(2, 5, dtype=torch.int32), ValueError),
                             (torch.zeros(5, dtype=torch.int32), ValueError), (torch.zeros(3, 4, dtype=torch.int32), ValueError),
                             (torch.zeros(3, 5, dtype=torch.int32), ValueError)):              # the last is on the host
        with pytest.raises(error):
            binding._positions(positions, rope, 5)


@pytest.mark.parametrize("interleaved", [False, True])
def test_one_axis_is_the_form_with_one(interleaved):
    r = np.random.default_rng(3)
    x, w, dy, pos, freq = r.normal(size=(5, 3, 16)), r.normal(size=16), r.normal(size=(5, 3, 16)), r.integers(0, 9000, 5), np.array([1, 0.1, 0.03])
    angle = ref.angles(np.stack((pos * 0 - 7, pos)), [1, 1, 1], freq)
    assert np.allclose(ref.heads(x, w, angle, 1e-3, interleaved), paged_ref.heads(x, w, pos, freq, 1e-3, interleaved))
    for a, b in zip(ref.heads_backward(dy, x, w, angle, 1e-3, interleaved), paged_ref.heads_backward(dy, x, w, pos, freq, 1e-3, interleaved)):
        assert np.allclose(a, b)


def test_each_pair_goes_by_its_own_axis():
    x = np.arange(8.0).reshape(1, 1, 8)
    angle = ref.angles([[np.pi / 2], [np.pi], [0.0]], [0, 1, 2], [1.0, 1.0, 1.0])
    assert np.allclose(ref.rotate(x, angle, True), [[[-1, 0, -2, -3, 4, 5, 6, 7]]])           # a quarter, a half, nothing, and what is not turned
    assert np.allclose(ref.rotate(x, angle, False), [[[-3, -1, 2, 0, -4, 5, 6, 7]]])


def test_angles_in_host_memory_are_refused():
    for axes in (None, [0, 1, 2, 0]):
        with pytest.raises(ValueError, match="rope must be on the device"):
            binding._heads(64, binding.Rope([1.0, 0.5, 0.25, 0.1], device="cpu", axes=axes), None, None, 1e-6)
