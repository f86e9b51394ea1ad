"""Pages of 8 bits: what is refused on the host before anything is launched (no device is touched), and the plain forms the GPU tests rest on."""
import ctypes
import os

import numpy as np
import pytest
import torch

import e4m3_ref as ref
from paper_2502_18394_amd import binding

FAKE, FAR, OUT, BIG = 1 << 20, 1 << 40, 1 << 41, 1 << 30        # never dereferenced: every call below fails its checks first


@pytest.fixture(scope="module")
def lib():
    from paper_2502_18394_amd import build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


def pool(**change):
    sizes = dict(layers=2, pages=8, Hkv=2, d=64, page=32, seqs=4, max_pages=5, dtype=binding.E4M3, k=FAR, v=FAR + BIG, book=FAKE, scales=FAKE)
    sizes.update(change)
    return ctypes.byref(binding.KvC(*sizes.values()))


def test_sizes_of_a_pool(lib):
    assert [lib.spectre_kv_bytes(pool(), w) for w in range(5)] == [2 * 8 * 2 * 32 * 64] * 2 + [4 * (8 + 4 + 8 + 20), 2 * 8 * 2 * 2 * 2 * 4, 0]
    assert lib.spectre_kv_bytes(pool(dtype=binding.BF16), 3) == 0
    assert lib.spectre_kv_bytes(pool(dtype=3), 0) == 0 and lib.spectre_kv_bytes(pool(dtype=5), 0) == 0
    # partial results and plans are those of bf16 rows
    a, b = (lib.spectre_kv_attend_workspace_bytes(pool(dtype=t), 3, 700, 8, 300, 5000, 0) for t in (binding.E4M3, binding.BF16))
    assert a == b > 0


@pytest.mark.parametrize("change,code", [(dict(scales=None), 1), (dict(scales=FAKE + 4), 1), (dict(k=FAR + 8), 1), (dict(d=32), 2), (dict(page=8), 2), (dict(dtype=2), 1)])
def test_pools_that_are_refused(lib, change, code):
    c = pool(**change)
    heads = ctypes.byref(binding.HeadsC(64, 64, 0, 1e-6, FAKE, FAKE, FAKE, 1, None))
    assert lib.spectre_kv_init(c, None) == code
    assert lib.spectre_kv_fork(c, FAKE, FAKE, 1, FAKE, BIG, None) == code
    assert lib.spectre_kv_compact(c, FAKE, BIG, None) == code and lib.spectre_kv_copy(c, FAKE, FAKE, 1, None) == code
    assert lib.spectre_kv_append(c, 0, heads, FAKE, 256, FAR, 128, FAR, 128, FAKE, None, 1, 3, 4, OUT, None) == code
    assert lib.spectre_kv_attend(c, 0, FAKE, 256, FAKE, None, 1, 1, 4, 1, 1, 0.1, 0, OUT, None, FAKE, BIG, None) == code


def test_rows_of_such_a_pool_are_bf16(lib):
    heads = ctypes.byref(binding.HeadsC(64, 64, 0, 1e-6, FAKE, FAKE, FAKE, 1, None))
    # a stride of 16 bytes of bf16, and no less
    assert lib.spectre_kv_append(pool(), 0, heads, FAKE, 260, FAR, 128, FAR, 128, FAKE, None, 1, 3, 4, OUT, None) == 1 and b"stride" in lib.spectre_last_error()
    assert lib.spectre_kv_attend(pool(), 0, FAKE, 260, FAKE, None, 1, 3, 4, 3, 9, 0.1, 0, OUT, None, FAKE, BIG, None) == 1
    # rows themselves are no pages
    assert lib.spectre_heads_forward(heads, FAKE, 256, FAR, 128, None, 3, 4, 2, binding.E4M3, OUT, OUT + BIG, None) == 1


def test_the_binding_refuses():
    k, v = torch.zeros(1, 2, 1, 4, 32, 16, dtype=torch.float8_e4m3fn), torch.zeros(1, 2, 1, 2, 64, 16, dtype=torch.float8_e4m3fn)
    book, scales = torch.zeros(8 + 1 + 2 + 3, dtype=torch.int32), torch.ones(1, 2, 1, 2, 2)
    for bad in (dict(scales=None), dict(scales=scales.double()), dict(scales=scales[:, :1]), dict(v=v.transpose(3, 4).contiguous()), dict(v=v.bfloat16())):
        a = dict(k=k, v=v, scales=scales)
        a.update(bad)
        with pytest.raises(ValueError):
            binding.KvPages(a["k"], a["v"], book, 1, 3, a["scales"])
    with pytest.raises(ValueError):                           # scales of pages that need none
        binding.KvPages(torch.zeros(1, 2, 1, 8, 16, 8, dtype=torch.bfloat16), torch.zeros(1, 2, 1, 2, 64, 8, dtype=torch.bfloat16), book, 1, 3, scales)


# ---------------------------------------------------------------- the plain forms
def test_codes_are_the_nearest_numbers():
    every = torch.arange(256, dtype=torch.uint8)
    x = ref.numbers(every).numpy()
    fine = np.isfinite(x)
    assert fine.sum() == 254 and x[fine].max() == ref.MOST
    assert np.array_equal(ref.code(x[fine]), every.numpy()[fine])
    assert np.array_equal(ref.code([np.nan, np.inf]) & 127, [127, 127])
    sizes = np.sort(x[fine & (np.arange(256) < 128)])
    r = np.random.default_rng(1)
    for y in np.concatenate((r.uniform(0, 448, 500), r.uniform(0, 0.05, 500), (sizes[1:] + sizes[:-1]) / 2)):
        got = ref.numbers(torch.from_numpy(ref.code([y]))).item()
        off = np.abs(sizes - y)
        assert abs(got - y) == off.min()
        if (off == off.min()).sum() == 2:
            assert int(ref.code([y])[0]) % 2 == 0             # halfway: the even one
    assert np.array_equal(ref.code(-sizes), ref.code(sizes) | 128)


def test_scales_are_the_smallest():
    for top in (448.0, 448.1, 1.75, 1.7500001, 3.4e38, 1e-3, 2.0 ** -120, 0.0):
        s = ref.scale_for([0.0, -top, np.inf, np.nan])
        assert top <= 448 * s and (s == 2.0 ** -100 or top > 448 * s / 2)
    assert ref.scale_for([1.75]) == 2.0 ** -8 and ref.scale_for([1.7500001]) == 2.0 ** -7


def test_a_larger_scale_leaves_codes_as_they_are():
    """But for subnormals: a normal code of the smaller scale is a number of the larger one, as long as it is a normal one there, too."""
    x = ref.numbers(torch.arange(126, dtype=torch.uint8)).numpy()
    for power in (1, 2, 5):
        y = x / 2.0 ** power
        again = ref.numbers(torch.from_numpy(ref.code(y))).numpy()
        assert np.array_equal(again[y >= 2.0 ** -6], y[y >= 2.0 ** -6]) and (np.abs(again - y) <= ref.SMALL).all()
