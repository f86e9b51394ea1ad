"""How much workspace an attention call asks for, and which batches are too large for a launch (no device is touched)."""
import ctypes
import subprocess
import sys

import pytest

from paper_2502_18394_amd import binding
from test_paged_refusals import FAKE, FAR, OUT, lib, pool  # noqa: F401

MB = 1 << 20


def test_an_empty_batch_has_a_plan(lib):  # noqa: F811
    """In a process of its own: a division by zero ends it."""
    code = ("import ctypes, sys; sys.path.insert(0, 'tests')\n"
            "from test_paged_refusals import pool\n"
            "from paper_2502_18394_amd import binding\n"
            "L = binding.lib()\n"
            "for d in (64, 128):\n"
            "    for dt in (0, 1):\n"
            "        c = ctypes.byref(pool(d=d, dtype=dt))\n"
            "        for B, T, new in ((0, 0, 1), (0, 0, 500), (3, 0, 1), (3, 0, 70), (1, 0, 4)):\n"
            "            assert 0 < L.spectre_kv_attend_workspace_bytes(c, B, T, 4, new, 300, 0) <= 4096, (B, T, new)\n")
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=__file__.rsplit("/", 2)[0])
    assert done.returncode == 0, (done.returncode, done.stderr[-500:])


def _sizes(lib, B, T, H, new, most, **change):
    c = pool(layers=1, pages=1 << 16, Hkv=8, page=64, seqs=4096, max_pages=1 << 14, **change)
    return lib.spectre_kv_attend_workspace_bytes(ctypes.byref(c), B, T, H, new, most, 0)


@pytest.mark.parametrize("d", [64, 128])
def test_workspaces_are_in_proportion(lib, d):  # noqa: F811
    size = lambda *a: _sizes(lib, *a, d=d)
    row = 4 * d + 8
    # a chunk beside decoding sequences, at the longest lengths; many ragged sequences; the chunk alone, of one length
    assert 0 < size(32, 8192 + 31, 32, 8192, 131072) < 512 * MB
    assert 0 < size(32, 2048 + 31, 32, 2048, 131072) < 300 * MB
    assert 0 < size(48, 60000, 32, 2000, 36000) < 60000 * 32 * (5 * row // 2 + 8) + 64 * MB
    assert 0 < size(1, 8192, 32, 8192, 131072) < 4 * MB
    # many single tokens of long sequences
    assert 0 < size(4096, 4096, 32, 1, 131072) < 300 * MB
    assert 0 < size(256, 256, 32, 1, 131072) < 300 * MB


@pytest.mark.parametrize("dtype", [binding.F32, binding.BF16])
def test_batches_too_large_for_a_launch(lib, dtype):  # noqa: F811
    """The call and the size query agree, before anything is launched; what can be launched with fewer parts is."""
    assert _sizes(lib, 256, 32768, 32, 32768, 131072, dtype=dtype) > 0
    c = ctypes.byref(pool(layers=1, pages=1 << 16, Hkv=8, page=64, seqs=4096, max_pages=1 << 14, dtype=dtype))
    B, T, new = 1024, 1 << 16, 1 << 16                      # 1024 tiles of 512 threads for each of 8192 pairs: 2^32 threads, one more than there can be
    assert lib.spectre_kv_attend_workspace_bytes(c, B, T, 32, new, 131072, 0) == 0
    assert lib.spectre_kv_attend(c, 0, FAKE, 2048, FAKE, None, B, T, 32, new, 131072, 0.1, 0, OUT, None, FAKE, 1 << 40, None) == 2
    assert lib.spectre_last_error()
