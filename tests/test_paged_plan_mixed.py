"""Parts of the single tokens beside a chunk of new tokens, as the workspace shows them (no device is touched)."""
import ctypes

import pytest

from paper_2502_18394_amd import binding
from test_paged_refusals import lib, pool  # noqa: F401


# sequences, tokens, heads, key heads, tokens of the chunk, keys -> parts: two workgroups a compute unit, of at least 256 keys each
CASES = [(2, 401, 32, 8, 400, 8192, 32), (3, 202, 1, 1, 200, 100000, 171), (2, 1001, 8, 4, 1000, 16000, 63), (6, 405, 16, 2, 400, 9000, 36)]


@pytest.mark.parametrize("dtype", [binding.F32, binding.BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,T,H,Hkv,new,most,parts", CASES)
def test_single_tokens_beside_a_chunk_have_their_parts(lib, B, T, H, Hkv, new, most, parts, d, dtype):  # noqa: F811
    c = ctypes.byref(pool(layers=1, pages=1 << 16, Hkv=Hkv, page=64, seqs=64, max_pages=1 << 14, d=d, dtype=dtype))
    got = lib.spectre_kv_attend_workspace_bytes(c, B, T, H, new, most, 0)
    # a place for each part of each row, d + 2 numbers, and how many there are; tiles have fewer parts here
    assert got == (T * H * (parts * (4 * d + 8) + 4) + 256) // 256 * 256
