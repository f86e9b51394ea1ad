"""How much workspace an attention call asks for (no device is touched)."""
import subprocess
import sys

from test_paged_refusals import lib  # noqa: F401


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
