"""What the paged attention calls refuse, on the host, before anything is launched (no device is touched), and the 64-bit forms that the GPU tests rest on."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paged_ref as ref
from paper_2502_18394_amd import binding

FAKE, FAR, OUT = 1 << 20, 1 << 40, 1 << 41        # never dereferenced: every call below fails its checks first


@pytest.fixture(scope="module")
def lib():
    from paper_2502_18394_amd import build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


def pool(**change):
    sizes = dict(layers=2, pages=8, Hkv=2, d=64, page=16, seqs=4, max_pages=5, dtype=binding.BF16, k=FAR, v=FAR + (1 << 30), book=FAKE)
    sizes.update(change)
    return binding.KvC(*sizes.values())


def said(lib, word):
    return word.encode() in lib.spectre_last_error()


def test_sizes_of_a_pool(lib):
    c = pool()
    assert [lib.spectre_kv_bytes(ctypes.byref(c), w) for w in range(3)] == [2 * 8 * 2 * 16 * 64 * 2] * 2 + [4 * (8 + 4 + 8 + 4 * 5)]
    assert lib.spectre_kv_bytes(ctypes.byref(pool(dtype=binding.F32)), 1) == 2 * 8 * 2 * 16 * 64 * 4
    assert lib.spectre_kv_bytes(ctypes.byref(c), 3) == 0 and lib.spectre_kv_bytes(None, 0) == 0
    assert lib.spectre_kv_workspace_bytes(ctypes.byref(c), 0) >= 4 * (3 * 8 + 8) and lib.spectre_kv_workspace_bytes(ctypes.byref(c), -1) == 0
    assert lib.spectre_kv_workspace_bytes(ctypes.byref(c), 100) >= 4 * (200 + 8)
    # more than 2^32 bytes
    assert lib.spectre_kv_bytes(ctypes.byref(pool(pages=1 << 20, Hkv=8, page=64)), 0) == 2 * (1 << 20) * 8 * 64 * 64 * 2


@pytest.mark.parametrize("change,code", [
    (dict(layers=0), 1), (dict(pages=-1), 1), (dict(Hkv=0), 1), (dict(seqs=0), 1), (dict(max_pages=0), 1), (dict(dtype=2), 1),
    (dict(d=32), 2), (dict(d=96), 2), (dict(page=8), 2), (dict(page=48), 2), (dict(page=512), 2), (dict(seqs=65537), 2), (dict(max_pages=(1 << 20) + 1), 2),
    (dict(k=None), 1), (dict(v=None), 1), (dict(book=None), 1), (dict(k=FAR + 8), 1), (dict(book=FAKE + 2), 1)])
def test_pools_that_are_refused(lib, change, code):
    c = ctypes.byref(pool(**change))
    big = 1 << 30
    assert lib.spectre_kv_init(c, None) == code
    assert lib.spectre_kv_reserve(c, FAKE, FAKE, 1, FAKE, big, None) == code
    assert lib.spectre_kv_fork(c, FAKE, FAKE, 1, FAKE, big, None) == code
    assert lib.spectre_kv_free(c, FAKE, 1, None) == code
    assert lib.spectre_kv_compact(c, FAKE, big, None) == code
    assert lib.spectre_kv_copy(c, FAKE, FAKE, 1, None) == code
    assert lib.spectre_kv_attend(c, 0, FAKE, 256, FAKE, None, 1, 1, 4, 1, 1, 0.1, 0, OUT, None, FAKE, big, None) == code
    assert lib.spectre_last_error()


def test_lists_and_workspaces_that_are_refused(lib):
    c = ctypes.byref(pool())
    big = 1 << 30
    for call in (lambda a, b, n, ws, size: lib.spectre_kv_reserve(c, a, b, n, ws, size, None), lambda a, b, n, ws, size: lib.spectre_kv_fork(c, a, b, n, ws, size, None)):
        assert call(None, FAKE, 1, FAKE, big) == 1 and call(FAKE, None, 1, FAKE, big) == 1 and call(FAKE, FAKE, -1, FAKE, big) == 1
        assert call(FAKE, FAKE, 1, None, big) == 3 and call(FAKE, FAKE, 1, FAKE, 16) == 3 and said(lib, "workspace")
        assert call(FAKE, FAKE, 1, FAKE + 4, big) == 1 and said(lib, "aligned")
        assert call(None, None, 0, None, 0) == 0                        # nothing to do
    assert lib.spectre_kv_fork(c, FAKE, FAKE, 5, FAKE, big, None) == 1  # more children than rows
    assert lib.spectre_kv_free(c, None, 1, None) == 1 and lib.spectre_kv_free(c, FAKE, -1, None) == 1 and lib.spectre_kv_free(c, None, 0, None) == 0
    assert lib.spectre_kv_copy(c, None, FAKE, 1, None) == 1 and lib.spectre_kv_copy(c, FAKE, FAKE, -2, None) == 1 and lib.spectre_kv_copy(c, None, None, 0, None) == 0
    assert lib.spectre_kv_compact(c, None, big, None) == 3 and lib.spectre_kv_compact(c, FAKE, 8, None) == 3


def heads(**change):
    P = dict(d=64, rot=64, interleaved=0, eps=1e-6, inv_freq=FAKE, wq=FAKE, wk=FAKE)
    P.update(change)
    return binding.HeadsC(*P.values())


ROW_ERRORS = [(dict(d=32), 2), (dict(rot=8), 2), (dict(rot=80), 2), (dict(rot=-16), 2), (dict(inv_freq=None), 1), (dict(wq=None), 1), (dict(wk=None), 1),
              (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(interleaved=2), 1)]


@pytest.mark.parametrize("change,code", ROW_ERRORS)
def test_head_parameters_that_are_refused(lib, change, code):
    P, big = ctypes.byref(heads(**change)), 1 << 30
    assert lib.spectre_heads_forward(P, FAKE, 256, FAR, 128, None, 3, 4, 2, 1, OUT, OUT + big, None) == code
    assert lib.spectre_heads_backward(P, FAKE, 256, FAR, 128, FAKE, 256, FAR, 128, None, 3, 4, 2, 1, OUT, OUT + big, FAKE, FAKE, FAKE, big, None) == code
    assert lib.spectre_kv_append(ctypes.byref(pool()), 0, P, FAKE, 256, FAR, 128, FAR, 128, FAKE, None, 1, 3, 4, OUT, None) == code


def test_rows_that_are_refused(lib):
    P, big = ctypes.byref(heads()), 1 << 30

    def forward(q=FAKE, qs=256, k=FAR, ks=128, T=3, H=4, Hkv=2, io=1, qo=OUT, ko=OUT + big):
        return lib.spectre_heads_forward(P, q, qs, k, ks, None, T, H, Hkv, io, qo, ko, None)

    for bad in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(q=FAKE + 8), dict(qs=255), dict(qs=260), dict(ks=64), dict(T=-1), dict(H=0),
                dict(Hkv=0), dict(io=3), dict(qo=FAKE), dict(qo=FAR + 256), dict(ko=OUT + 512), dict(ks=-128)):
        assert forward(**bad) == 1, bad
    assert forward(T=0, q=None, k=None) == 0
    assert lib.spectre_heads_forward(None, FAKE, 256, FAR, 128, None, 3, 4, 2, 1, OUT, OUT + big, None) == 1
    assert lib.spectre_heads_backward_workspace_bytes(0, 64) == 0 and lib.spectre_heads_backward_workspace_bytes(9, 32) == 0
    need = lib.spectre_heads_backward_workspace_bytes(3, 64)
    assert need >= 2 * 64 * 8

    def backward(gq=OUT, gk=OUT + big, gwq=FAKE, gwk=FAKE, ws=FAKE, size=need, dq=FAKE):
        return lib.spectre_heads_backward(P, dq, 256, FAR, 128, FAKE, 256, FAR, 128, None, 3, 4, 2, 1, gq, gk, gwq, gwk, ws, size, None)

    for bad, code in ((dict(gq=None), 1), (dict(gk=FAR), 1), (dict(gwq=None), 1), (dict(gwk=None), 1), (dict(ws=None), 3), (dict(size=need - 256), 3), (dict(dq=None), 1)):
        assert backward(**bad) == code, bad


def test_batches_that_are_refused(lib):
    c, P, big = ctypes.byref(pool()), ctypes.byref(heads()), 1 << 30

    def append(layer=0, q=FAKE, qs=256, start=FAKE, B=2, T=3, H=4, out=OUT, k=FAR):
        return lib.spectre_kv_append(c, layer, P, q, qs, k, 128, FAR, 128, start, None, B, T, H, out, None)

    for bad in (dict(layer=2), dict(layer=-1), dict(start=None), dict(B=0), dict(B=5), dict(T=-1), dict(H=3), dict(H=0), dict(q=None), dict(out=None), dict(qs=128),
                dict(out=FAKE), dict(k=FAR + 4)):
        assert append(**bad) == 1, bad
    assert append(T=0, q=None) == 0 and append(T=0, B=0, q=None) == 0
    assert lib.spectre_kv_append(c, 0, ctypes.byref(heads(d=128, rot=0)), FAKE, 256, FAR, 128, FAR, 128, FAKE, None, 1, 3, 4, OUT, None) == 1

    def attend(layer=0, q=FAKE, qs=256, start=FAKE, B=2, T=3, H=4, new=3, most=300, scale=0.125, window=0, out=OUT, ws=FAKE, size=big):
        return lib.spectre_kv_attend(c, layer, q, qs, start, None, B, T, H, new, most, scale, window, out, None, ws, size, None)

    for bad, code in ((dict(layer=5), 1), (dict(start=None), 1), (dict(B=0), 1), (dict(B=7), 1), (dict(H=5), 1), (dict(new=0), 1), (dict(most=0), 1), (dict(window=-1), 1),
                      (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(q=None), 1), (dict(out=None), 1),
                      (dict(out=FAKE + 16), 1), (dict(qs=250), 1), (dict(ws=None), 3), (dict(size=64), 3), (dict(new=1 << 30), 2), (dict(T=-2), 1)):
        assert attend(**bad) == code, bad
    assert attend(T=0, q=None, out=None, ws=None) == 0 and attend(T=0, B=0, q=None, out=None, ws=None) == 0
    assert attend(scale=1e-31) == 1 and attend(scale=1e31) == 1
    assert attend(T=1 << 29, B=4, H=4, new=1) == 2                       # more rows than an int counts
    assert lib.spectre_kv_attend_workspace_bytes(c, 2, 3, 5, 3, 300, 0) == 0
    assert lib.spectre_kv_attend_workspace_bytes(c, 2, 3, 4, 3, 300, 0) > 3 * 4 * 64 * 4


def test_the_binding_refuses_what_is_not_on_the_device():
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.qk_norm_rotate(x, x)
    with pytest.raises(TypeError):
        binding.qk_norm_rotate(x.half(), x.half())
    with pytest.raises(ValueError):
        binding.KvPages(torch.zeros(1, 2, 1, 8, 16, 4, dtype=torch.bfloat16), None, None, 1, 1)
    with pytest.raises(binding.SpectreError):
        binding.KvPages.empty(1, 4, 2, 80, 16, 2, 2)


# ---------------------------------------------------------------- the plain forms
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_formula_against_differences(interleaved):
    r = np.random.default_rng(1)
    x, w, dy, pos = r.normal(size=(3, 2, 8)), r.normal(size=8), r.normal(size=(3, 2, 8)), np.array([0, 7, 90000])
    freq = np.array([1.0, 0.1, 0.01])                                    # six of eight channels
    gx, gw = ref.heads_backward(dy, x, w, pos, freq, 1e-3, interleaved)
    loss = lambda x, w: (ref.heads(x, w, pos, freq, 1e-3, interleaved) * dy).sum()
    h = 1e-6
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - gx[i]) < 1e-7
    for i in range(8):
        e = np.zeros_like(w)
        e[i] = h
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - gw[i]) < 1e-7


def test_rotation_keeps_lengths_and_depends_on_distance():
    r = np.random.default_rng(2)
    q, k, freq = r.normal(size=(1, 1, 8)), r.normal(size=(1, 1, 8)), np.array([1.0, 0.3, 0.09, 0.01])
    at = lambda x, p: ref.rotate(x, np.array([p]), freq, False)[0, 0]
    assert np.allclose(np.linalg.norm(at(q, 12345)), np.linalg.norm(q))
    assert np.allclose(at(q, 10) @ at(k, 3), at(q, 1007) @ at(k, 1000)) and not np.allclose(at(q, 10) @ at(k, 3), at(q, 10) @ at(k, 4))


def test_attention_form_at_its_borders():
    r = np.random.default_rng(3)
    q, k, v = r.normal(size=(3, 4, 8)), r.normal(size=(5, 2, 8)), r.normal(size=(5, 2, 8))
    out, lse = ref.attend(q, k, v, 0.5)
    s = 0.5 * k[:, 1] @ q[2, 3]                                          # the last query sees every key, head 3 reads key head 1
    assert np.allclose(out[2, 3], np.exp(s) @ v[:, 1] / np.exp(s).sum()) and np.allclose(lse[2, 3], np.log(np.exp(s).sum()))
    one, _ = ref.attend(q, k, v, 0.5, window=1)
    assert np.allclose(one[0, 0], v[2, 0]) and np.allclose(one[2, 2], v[4, 1])
    none, lse = ref.attend(q, k[:2], v[:2], 0.5)                          # more queries than tokens
    assert (none[0] == 0).all() and np.isneginf(lse[0]).all() and np.allclose(none[1, 0], v[0, 0])
    gone, _ = ref.attend(q, k, v, 0.5, there=np.array([True, False, True, True, True]))
    assert np.allclose(gone[2, 0], ref.attend(q[2:], np.delete(k, 1, 0), np.delete(v, 1, 0), 0.5)[0][0, 0])


def test_plain_bookkeeping_keeps_count():
    b = ref.Book(4, 10, 4, 16)
    b.reserve([0, 1], [40, 16])
    assert b.table[0][:3] == [0, 1, 2] and b.table[1][0] == 3 and b.lens == [40, 16, 0, 0]
    assert b.fork([0], [2]) == [(2, 4, 8)] and b.refs[:5] == [2, 2, 1, 1, 1] and b.table[2][:3] == [0, 1, 4]
    b.free([0, 1])
    assert b.refs[:5] == [1, 1, 0, 0, 1] and b.compact() == [(4, 2)] and b.table[2] == [0, 1, 2, -1] and b.status[1:3] == [1, 3]
