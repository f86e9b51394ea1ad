"""Thin Python binding of the C ABI in ``include/spectre.h``.

Argument marshalling only: torch supplies device memory and the current stream,
every step of the computation runs in the HIP library.  There is no fallback: if
``libspectre_hip.so`` has not been built (``python -m paper_2502_18394_amd.build``)
the first call raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspectre_hip.so")

F32, BF16, E4M3 = 0, 1, 4
READ_NEWEST, READ_WINDOW = 0, 1
OK, EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP, ENOTREADY = 0, 1, 2, 3, 4, 5
OPT_LANES, OPT_SCRATCH_MB, OPT_FUSED_4096, OPT_SLAB_COMPILE_TIME, OPT_HEAD_AFFINE, OPT_GROUPS, OPT_LANE_SHUFFLES = 0, 1, 2, 3, 4, 5, 6
MIX_BF16_SCRATCH = 1

_lib = None


class SpectreError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"spectre status {code}: {msg}")
        self.code = code


class GateParamsC(ctypes.Structure):
    _fields_ = [("Hg", ctypes.c_int), ("d", ctypes.c_int), ("d_g", ctypes.c_int), ("n_fft", ctypes.c_int),
                ("ln_gamma", ctypes.c_void_p), ("ln_beta", ctypes.c_void_p), ("ln_eps", ctypes.c_float),
                ("W1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("W2", ctypes.c_void_p), ("b2", ctypes.c_void_p),
                ("modrelu_bias", ctypes.c_void_p), ("toeplitz", ctypes.c_void_p), ("toeplitz_r", ctypes.c_int)]


class WrmParamsC(ctypes.Structure):
    _fields_ = [("Hg", ctypes.c_int), ("d", ctypes.c_int), ("d_w", ctypes.c_int), ("levels", ctypes.c_int),
                ("ln_gamma", ctypes.c_void_p), ("ln_beta", ctypes.c_void_p), ("ln_eps", ctypes.c_float),
                ("W1", ctypes.c_void_p), ("b1", ctypes.c_void_p), ("W2", ctypes.c_void_p), ("b2", ctypes.c_void_p)]


class PrefixCacheC(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("H", ctypes.c_int), ("d", ctypes.c_int), ("N_max", ctypes.c_int),
                ("N_mem", ctypes.c_int), ("t", ctypes.c_longlong),
                ("prefix_fft", ctypes.c_void_p), ("v_buf", ctypes.c_void_p), ("q_buf", ctypes.c_void_p),
                ("sum_q", ctypes.c_void_p), ("twiddle", ctypes.c_void_p),
                ("pending", ctypes.c_void_p), ("pending_cap", ctypes.c_int), ("n_pending", ctypes.c_int),
                ("pending_slot", ctypes.c_int * 32)]


class KvC(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int), ("pages", ctypes.c_int), ("Hkv", ctypes.c_int), ("d", ctypes.c_int), ("page", ctypes.c_int),
                ("seqs", ctypes.c_int), ("max_pages", ctypes.c_int), ("dtype", ctypes.c_int), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("book", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


class HeadsC(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int), ("rot", ctypes.c_int), ("interleaved", ctypes.c_int), ("eps", ctypes.c_float),
                ("inv_freq", ctypes.c_void_p), ("wq", ctypes.c_void_p), ("wk", ctypes.c_void_p), ("axes", ctypes.c_int), ("axis", ctypes.c_void_p)]


def lib():
    """The loaded C library; raises if it is missing (never falls back to another path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2502_18394_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        L.spectre_last_error.restype = ctypes.c_char_p
        for name in ("spectre_gate_workspace_bytes", "spectre_mix_workspace_bytes", "spectre_prefix_bytes",
                     "spectre_project_workspace_bytes", "spectre_wrm_gates_workspace_bytes",
                     "spectre_wrm_apply_workspace_bytes",
                     "spectre_prefix_update_workspace_bytes", "spectre_prefix_readout_workspace_bytes",
                     "spectre_prefix_step_workspace_bytes", "spectre_prefix_set_memory_workspace_bytes",
                     "spectre_mix_static_bytes", "spectre_layer_workspace_bytes", "spectre_kv_bytes", "spectre_kv_workspace_bytes",
                     "spectre_kv_attend_workspace_bytes", "spectre_heads_backward_workspace_bytes", "spectre_norm_backward_workspace_bytes"):
            getattr(L, name).restype = ctypes.c_size_t
        L.spectre_get_option.restype = ctypes.c_long
        # with the types declared, ctypes converts plain integers itself: a wrapper object per argument costs a few
        # microseconds a call, as much as the kernels of the smallest ones take
        p, i, n, f, ll = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_double, ctypes.c_longlong
        for name, types in {
                "spectre_mix_workspace_bytes": (i, i, i, i, i),
                "spectre_mix_forward_ex": (p, p, p, i, i, i, i, i, ctypes.c_uint, p, n, p),
                "spectre_gate_workspace_bytes": (i, i, i, p),
                "spectre_gate": (p, i, i, f, p, i, i, i, ctypes.c_longlong, p, p, n, p),
                "spectre_layer_workspace_bytes": (i, i, i, i, i, p, p),
                "spectre_layer_forward": (p, p, p, i, p, p, p, i, i, i, i, i, p, n, p),
                "spectre_prefix_init": (p, p), "spectre_prefix_flush": (p, p),
                "spectre_prefix_update_workspace_bytes": (p, i, i),
                "spectre_prefix_update": (p, p, p, i, i, p, n, p),
                "spectre_prefix_readout_workspace_bytes": (p, i, i),
                "spectre_prefix_readout": (p, p, i, p, i, p, n, p),
                "spectre_prefix_step_workspace_bytes": (p, p),
                "spectre_prefix_step": (p, p, p, p, p, i, p, n, p),
                "spectre_kv_bytes": (p, i), "spectre_kv_workspace_bytes": (p, i), "spectre_kv_prepare": (), "spectre_kv_init": (p, p),
                "spectre_kv_reserve": (p, p, p, i, p, n, p), "spectre_kv_fork": (p, p, p, i, p, n, p), "spectre_kv_free": (p, p, i, p),
                "spectre_kv_compact": (p, p, n, p), "spectre_kv_copy": (p, p, p, i, p),
                "spectre_heads_forward": (p, p, ll, p, ll, p, i, i, i, i, p, p, p),
                "spectre_heads_backward_workspace_bytes": (i, i),
                "spectre_heads_backward": (p, p, ll, p, ll, p, ll, p, ll, p, i, i, i, i, p, p, p, p, p, n, p),
                "spectre_kv_append": (p, i, p, p, ll, p, ll, p, ll, p, p, i, i, i, p, p),
                "spectre_kv_append_at": (p, i, p, p, ll, p, ll, p, ll, p, p, p, i, i, i, p, p),
                "spectre_norm_forward": (p, ll, p, ll, p, i, i, ctypes.c_float, i, p, p, i, p, p),
                "spectre_norm_backward_workspace_bytes": (i, i, i),
                "spectre_norm_backward": (p, ll, p, ll, p, ll, p, i, i, ctypes.c_float, i, p, p, p, n, p),
                "spectre_kv_attend_workspace_bytes": (p, i, i, i, i, i, i),
                "spectre_kv_attend": (p, i, p, ll, p, p, i, i, i, i, i, ctypes.c_float, i, p, p, p, n, p)}.items():
            getattr(L, name).argtypes = types
        _lib = L
    return _lib


def _check(rc):
    if rc != OK:
        raise SpectreError(rc, lib().spectre_last_error().decode())


def _dtype_code(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t, name):
    """Address of a contiguous device tensor, for the functions whose argument types are declared."""
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous device tensor")
    return t.data_ptr()


def _dev(t, name):
    """The same for the others."""
    return ctypes.c_void_p(_ptr(t, name))


def _raw_stream(stream):
    """Handle of `stream`, or of the current one (without the Stream object that torch.cuda.current_stream builds), as a plain integer, for
    the functions whose argument types are declared."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _stream(stream):
    """The same for the others."""
    return ctypes.c_void_p(_raw_stream(stream))


def _given(ws):
    """(address, bytes) of the caller's workspace from its first 256-byte boundary on."""
    at = _ptr(ws, "ws")
    off = -at % 256
    return at + off, max(0, ws.numel() * ws.element_size() - off)


def _workspace(nbytes, device, ws):
    nbytes = max(int(nbytes), 256)
    size = 0 if ws is None else ws.numel() * ws.element_size()
    if size < nbytes:
        size = nbytes + 256
        ws = torch.empty(size, dtype=torch.uint8, device=device)
    at = _ptr(ws, "ws")
    off = -at % 256
    return ws, ctypes.c_void_p(at + off), ctypes.c_size_t(size - off)


def version():
    return int(lib().spectre_version())


def length_supported(n, d):
    return bool(lib().spectre_length_supported(ctypes.c_int(n), ctypes.c_int(d)))


_prepared = set()


def prepare(n, d=64):
    """Set-up for transform length n on the current device (tables, helper stream): the library's one call that
    allocates and synchronises.  The functions below call it the first time they see a length."""
    key = (torch.cuda.current_device(), int(n), int(d))
    if key not in _prepared:
        _check(lib().spectre_prepare(ctypes.c_int(n), ctypes.c_int(d)))
        _prepared.add(key)


def shutdown():
    """Free the library's tables and helper streams; lengths are prepared again on their next use."""
    lib().spectre_shutdown()
    _prepared.clear()


def set_option(which, value):
    """Tuning switch `which` (one of the OPT_* constants) := value; value < 0 restores the default."""
    _check(lib().spectre_set_option(ctypes.c_int(which), ctypes.c_long(value)))


def get_option(which):
    return int(lib().spectre_get_option(ctypes.c_int(which)))


def mix_workspace_bytes(B, L, H, d, io):
    return lib().spectre_mix_workspace_bytes(B, L, H, d, io)


def mix_forward(v, g, out=None, ws=None, stream=None, flags=0):
    """out[b,:,h,c] = irfft_L(g[b,h,:] * rfft_L(v[b,:,h,c])); v [B,L,H,d] f32/bf16, g complex64 [B,H,L//2+1].
    flags: 0 or MIX_BF16_SCRATCH (see spectre_mix_forward_ex)."""
    B, L, H, d = v.shape
    prepare(L, d)
    io = _dtype_code(v)
    if g.dtype != torch.complex64 or g.shape != (B, H, L // 2 + 1):
        raise ValueError("g must be complex64 [B,H,L//2+1]")
    if out is None:
        out = torch.empty_like(v)
    args = (_ptr(v, "v"), _ptr(g, "g"), _ptr(out, "out"), B, L, H, d, io, flags)
    st = _raw_stream(stream)
    if ws is not None:                     # the library checks its size; asking for the size first is a call of its own
        rc = lib().spectre_mix_forward_ex(*args, *_given(ws), st)
        if rc != EWORKSPACE:
            _check(rc)
            return out
    ws, wsp, wsn = _workspace(mix_workspace_bytes(B, L, H, d, io), v.device, ws)
    _check(lib().spectre_mix_forward_ex(*args, wsp, wsn, st))
    return out


def mix_forward_static(v, g, out=None, stream=None):
    """mix_forward on the library's built-in scratch array: no workspace, no allocation inside the call
    (spectre_mix_forward_static; four-step lengths, B*H*L <= 4 Mi)."""
    B, L, H, d = v.shape
    if g.dtype != torch.complex64 or tuple(g.shape) != (B, H, L // 2 + 1):
        raise ValueError("g must be complex64 [B,H,L//2+1]")
    if out is None:
        out = torch.empty_like(v)
    _check(lib().spectre_mix_forward_static(_dev(v, "v"), _dev(g, "g"), _dev(out, "out"), ctypes.c_int(B),
                                            ctypes.c_int(L), ctypes.c_int(H), ctypes.c_int(d),
                                            ctypes.c_int(_dtype_code(v)), _stream(stream)))
    return out


def project(x, Wq, Wv, want_q=False, want_sum_q=True, ws=None, stream=None):
    """Per-head token projection (Eq. 2).  x [B,L,H,64] f32/bf16; Wq, Wv float32 [Hw,64,64] (Hw = H or 1).
    Returns (v, q or None, sum_q float64 [B,H,64] or None)."""
    B, L, H, d = x.shape
    io = _dtype_code(x)
    for w in (Wq, Wv):
        if w.dtype != torch.float32 or tuple(w.shape[1:]) != (d, d) or w.shape[0] != Wq.shape[0]:
            raise ValueError("Wq, Wv must be float32 [Hw,d,d]")
    v = torch.empty_like(x)
    q = torch.empty_like(x) if want_q else None
    sq = torch.empty((B, H, d), dtype=torch.float64, device=x.device) if want_sum_q else None
    need = lib().spectre_project_workspace_bytes(ctypes.c_int(B), ctypes.c_int(L), ctypes.c_int(H), ctypes.c_int(d))
    ws, wsp, wsn = _workspace(need, x.device, ws)
    _check(lib().spectre_project(_dev(x, "x"), _dev(Wq, "Wq"), _dev(Wv, "Wv"), ctypes.c_int(Wq.shape[0]),
                                 ctypes.c_int(B), ctypes.c_int(L), ctypes.c_int(H), ctypes.c_int(d), ctypes.c_int(io),
                                 _dev(v, "v"), None if q is None else _dev(q, "q"),
                                 None if sq is None else _dev(sq, "sum_q"), wsp, wsn, _stream(stream)))
    return v, q, sq


class GateParams:
    """Device copies of the gate parameters plus the C parameter block.

    ``params`` uses the paper's row-vector convention (hid = qbar W1, u = hid W2) with
    W1 [Hg,d,d_g] and W2 [Hg,d_g,2F]; the library wants W2 output-major, [Hg,2F,d_g], so it is
    transposed once here while it is copied to the device."""

    def __init__(self, params, device="cuda"):
        def dev(a):
            return None if a is None else torch.as_tensor(a, dtype=torch.float32).to(device).contiguous()
        self.t = {k: dev(params[k]) for k in ("ln_gamma", "ln_beta", "W1", "b1", "b2")}
        self.t["modrelu_bias"] = dev(params.get("modrelu_bias"))
        Hg, d, d_g = self.t["W1"].shape
        self.n_fft = int(params["n_fft"])
        F = self.n_fft // 2 + 1
        w2 = torch.as_tensor(params["W2"], dtype=torch.float32).to(device)
        assert tuple(w2.shape) == (Hg, d_g, 2 * F)
        self.t["W2"] = w2.transpose(1, 2).contiguous()
        del w2
        self.Hg, self.d, self.d_g, self.F = Hg, d, d_g, F
        taps = params.get("toeplitz")
        self.t["toeplitz"], r = None, 0
        if taps is not None:
            taps = torch.as_tensor(taps).to(torch.complex64).to(device).contiguous()
            assert taps.ndim == 2 and taps.shape[0] == Hg and taps.shape[1] % 2 == 1
            self.t["toeplitz"], r = taps, taps.shape[1] // 2
        p = lambda k: None if self.t[k] is None else ctypes.c_void_p(self.t[k].data_ptr())
        self.c = GateParamsC(Hg, d, d_g, self.n_fft, p("ln_gamma"), p("ln_beta"), float(params["ln_eps"]),
                             p("W1"), p("b1"), p("W2"), p("b2"), p("modrelu_bias"), p("toeplitz"), r)


def gate_workspace_bytes(B, L, H, P):
    return lib().spectre_gate_workspace_bytes(B, L, H, ctypes.byref(P.c))


def gate(q, P, inv_count, pooled=False, phase_pos=0, g_out=None, ws=None, stream=None):
    """Spectral gate complex64 [B,H,F].  q: query rows [B,L,H,d] (f32/bf16), or with pooled=True
    their sum over positions as float64 [B,H,d]."""
    if pooled:
        if q.dtype != torch.float64:
            raise TypeError("pooled q must be float64 [B,H,d]")
        B, H, d = q.shape
        L, code = 1, F32
    else:
        B, L, H, d = q.shape
        code = _dtype_code(q)
    if d != P.d:
        raise ValueError("d mismatch")
    if g_out is None:
        g_out = torch.empty((B, H, P.F), dtype=torch.complex64, device=q.device)
    args = (_ptr(q, "q"), 1 if pooled else 0, code, inv_count, ctypes.byref(P.c), B, L, H, int(phase_pos), _ptr(g_out, "g_out"))
    st = _raw_stream(stream)
    if ws is not None:                     # as in mix_forward
        rc = lib().spectre_gate(*args, *_given(ws), st)
        if rc != EWORKSPACE:
            _check(rc)
            return g_out
    ws, wsp, wsn = _workspace(gate_workspace_bytes(B, L, H, P), q.device, ws)
    _check(lib().spectre_gate(*args, wsp, wsn, st))
    return g_out


class WrmParams:
    """Device copies of the wavelet-refinement MLP (Sec. 3.5 step b) plus the C parameter block.
    W1 [Hg,d,d_w], b1 [Hg,d_w], W2 [Hg,d_w,(levels+1)*d], b2 [Hg,(levels+1)*d]."""

    def __init__(self, params, device="cuda"):
        self.t = {k: torch.as_tensor(params[k], dtype=torch.float32).to(device).contiguous()
                  for k in ("ln_gamma", "ln_beta", "W1", "b1", "W2", "b2")}
        Hg, d, d_w = self.t["W1"].shape
        self.levels = int(params["levels"])
        assert tuple(self.t["W2"].shape) == (Hg, d_w, (self.levels + 1) * d)
        self.Hg, self.d, self.d_w = Hg, d, d_w
        p = lambda k: ctypes.c_void_p(self.t[k].data_ptr())
        self.c = WrmParamsC(Hg, d, d_w, self.levels, p("ln_gamma"), p("ln_beta"), float(params["ln_eps"]),
                            p("W1"), p("b1"), p("W2"), p("b2"))


def wrm_gates(q, P, inv_count, pooled=False, s_out=None, ws=None, stream=None):
    """Level gates float32 [B,H,levels+1,d] from query rows [B,L,H,d] or (pooled=True) their float64 sum [B,H,d]."""
    if pooled:
        if q.dtype != torch.float64:
            raise TypeError("pooled q must be float64 [B,H,d]")
        B, H, d = q.shape
        L, code = 1, F32
    else:
        B, L, H, d = q.shape
        code = _dtype_code(q)
    if d != P.d:
        raise ValueError("d mismatch")
    if s_out is None:
        s_out = torch.empty((B, H, P.levels + 1, d), dtype=torch.float32, device=q.device)
    need = lib().spectre_wrm_gates_workspace_bytes(ctypes.c_int(B), ctypes.c_int(L), ctypes.c_int(H), ctypes.byref(P.c))
    ws, wsp, wsn = _workspace(need, q.device, ws)
    _check(lib().spectre_wrm_gates(_dev(q, "q"), ctypes.c_int(1 if pooled else 0), ctypes.c_int(code),
                                   ctypes.c_double(inv_count), ctypes.byref(P.c), ctypes.c_int(B), ctypes.c_int(L),
                                   ctypes.c_int(H), _dev(s_out, "s_out"), wsp, wsn, _stream(stream)))
    return s_out


def wrm_apply_workspace_bytes(B, L, H, d, levels):
    return int(lib().spectre_wrm_apply_workspace_bytes(ctypes.c_int(B), ctypes.c_int(L), ctypes.c_int(H),
                                                       ctypes.c_int(d), ctypes.c_int(levels)))


def wrm_apply(v, s, out=None, ws=None, stream=None):
    """v + iDWT(s * DWT(v)) along the sequence axis (Sec. 3.5 steps a, c, d); v [B,L,H,d] f32/bf16,
    s float32 [B,H,levels+1,d].  Pass out=v for in-place operation."""
    B, L, H, d = v.shape
    if s.dtype != torch.float32 or s.ndim != 4 or tuple(s.shape[:2]) != (B, H) or s.shape[3] != d:
        raise ValueError("s must be float32 [B,H,levels+1,d]")
    levels = s.shape[2] - 1
    if out is None:
        out = torch.empty_like(v)
    ws, wsp, wsn = _workspace(wrm_apply_workspace_bytes(B, L, H, d, levels), v.device, ws)
    _check(lib().spectre_wrm_apply(_dev(v, "v"), _dev(s, "s"), _dev(out, "out"), ctypes.c_int(B), ctypes.c_int(L),
                                   ctypes.c_int(H), ctypes.c_int(d), ctypes.c_int(levels),
                                   ctypes.c_int(_dtype_code(v)), wsp, wsn, _stream(stream)))
    return out


def wrm_apply_coeff(v, s, levels, out=None, ws=None, stream=None):
    """v + iDWT(s * DWT(v)) with one gate per wavelet coefficient and channel: v [B,L,H,d] f32/bf16,
    s float32 [B,H,L,d] in the analysis' coefficient order [a_J | d_J | ... | d_1]."""
    B, L, H, d = v.shape
    if s.dtype != torch.float32 or tuple(s.shape) != (B, H, L, d):
        raise ValueError("s must be float32 [B,H,L,d]")
    if out is None:
        out = torch.empty_like(v)
    ws, wsp, wsn = _workspace(wrm_apply_workspace_bytes(B, L, H, d, levels), v.device, ws)
    _check(lib().spectre_wrm_apply_coeff(_dev(v, "v"), _dev(s, "s"), _dev(out, "out"), ctypes.c_int(B), ctypes.c_int(L),
                                         ctypes.c_int(H), ctypes.c_int(d), ctypes.c_int(levels),
                                         ctypes.c_int(_dtype_code(v)), wsp, wsn, _stream(stream)))
    return out


def layer_forward(x, Wq, Wv, P, W=None, out=None, ws=None, stream=None):
    """The whole layer in one call (spectre_layer_forward): projection, pooled query, gate, mixer and, with W (a
    WrmParams), the wavelet refinement.  x [B,L,H,64] f32/bf16; Wq, Wv float32 [Hw,64,64]; P a GateParams for L."""
    B, L, H, d = x.shape
    io = _dtype_code(x)
    prepare(L, d)
    if out is None:
        out = torch.empty_like(x)
    wc = ctypes.byref(W.c) if W is not None else None
    need = lib().spectre_layer_workspace_bytes(B, L, H, d, io, ctypes.byref(P.c), wc)
    if need == 0:
        raise SpectreError(EUNSUPPORTED, lib().spectre_last_error().decode())
    ws, wsp, wsn = _workspace(need, x.device, ws)
    _check(lib().spectre_layer_forward(_ptr(x, "x"), _ptr(Wq, "Wq"), _ptr(Wv, "Wv"), Wq.shape[0], ctypes.byref(P.c), wc,
                                       _ptr(out, "out"), B, L, H, d, io, wsp, wsn, _stream(stream)))
    return out


class PrefixCache:
    """Caller-owned Prefix-FFT cache state (Algorithm 1) in device memory."""

    def __init__(self, B, H, d, N_max, N_mem=0, defer=0, device="cuda"):
        """N_max = ring capacity; N_mem = persistent memory rows (Sec. 3.4); n = N_mem + N_max is the transform length.
        defer > 0: step() leaves up to `defer` rank-one updates pending and only reads the cache (see spectre.h)."""
        L = lib()
        n = N_max + N_mem
        self.B, self.H, self.d, self.N, self.N_mem, self.n = B, H, d, N_max, N_mem, n
        self.F = n // 2 + 1
        nb = [int(L.spectre_prefix_bytes(ctypes.c_int(B), ctypes.c_int(H), ctypes.c_int(d), ctypes.c_int(n),
                                         ctypes.c_int(w))) for w in range(5)]
        if min(nb) == 0:
            raise SpectreError(EUNSUPPORTED, f"no prefix cache for B={B} H={H} d={d} N_mem+N_max={n}")
        self.prefix_fft = torch.empty((B, H, self.F, d), dtype=torch.complex64, device=device)
        self.v_buf = torch.empty((B, H, n, d), dtype=torch.float32, device=device)
        self.q_buf = torch.empty((B, H, n, d), dtype=torch.float32, device=device)
        self.sum_q = torch.empty((B, H, d), dtype=torch.float64, device=device)
        self.twiddle = torch.empty((n,), dtype=torch.complex64, device=device)
        for t, nbytes in zip((self.prefix_fft, self.v_buf, self.q_buf, self.sum_q, self.twiddle), nb):
            assert t.numel() * t.element_size() == nbytes, (t.shape, nbytes)
        self.pending = torch.zeros((defer, B, H, d), dtype=torch.float32, device=device) if defer > 0 else None
        self.c = PrefixCacheC(B, H, d, N_max, N_mem, 0, self.prefix_fft.data_ptr(), self.v_buf.data_ptr(),
                              self.q_buf.data_ptr(), self.sum_q.data_ptr(), self.twiddle.data_ptr(),
                              self.pending.data_ptr() if defer > 0 else None, defer, 0)
        self._ws = None
        _check(L.spectre_prefix_init(ctypes.byref(self.c), _stream(None)))

    def reset(self, stream=None):
        """Back to the empty cache (t = 0, zero state); memory rows, if any, must be set again."""
        self.c.n_pending = 0
        _check(lib().spectre_prefix_init(ctypes.byref(self.c), _stream(stream)))

    def set_memory(self, mem, stream=None):
        """mem float32 [1 or B, H, N_mem, d]: the persistent memory rows; call once, before any token."""
        if mem.dtype != torch.float32 or mem.ndim != 4 or tuple(mem.shape[1:]) != (self.H, self.N_mem, self.d):
            raise ValueError("mem must be float32 [1 or B, H, N_mem, d]")
        prepare(self.n, self.d)
        need = lib().spectre_prefix_set_memory_workspace_bytes(ctypes.byref(self.c))
        self._ws, wsp, wsn = _workspace(need, mem.device, self._ws)
        _check(lib().spectre_prefix_set_memory(ctypes.byref(self.c), _dev(mem, "mem"), ctypes.c_int(mem.shape[0]),
                                               wsp, wsn, _stream(stream)))

    @property
    def t(self):
        return int(self.c.t)

    @property
    def n_pending(self):
        return int(self.c.n_pending)

    def flush(self, stream=None):
        """Apply the pending deferred updates to prefix_fft."""
        _check(lib().spectre_prefix_flush(ctypes.byref(self.c), _stream(stream)))

    def update(self, v_new, q_new, stream=None):
        B, T, H, d = v_new.shape
        assert (B, H, d) == (self.B, self.H, self.d) and q_new.shape == v_new.shape and q_new.dtype == v_new.dtype
        io = _dtype_code(v_new)
        prepare(self.n, self.d)
        need = lib().spectre_prefix_update_workspace_bytes(ctypes.byref(self.c), T, io)
        self._ws, wsp, wsn = _workspace(need, v_new.device, self._ws)
        _check(lib().spectre_prefix_update(ctypes.byref(self.c), _ptr(v_new, "v_new"), _ptr(q_new, "q_new"), T, io, wsp,
                                           wsn, _stream(stream)))

    def readout(self, g, mode=READ_NEWEST, dtype=torch.float32, stream=None):
        io = F32 if dtype == torch.float32 else BF16
        prepare(self.n, self.d)
        rows = 1 if mode == READ_NEWEST else min(self.t, self.N)
        out = torch.empty((self.B, rows, self.H, self.d), dtype=dtype, device=g.device)
        need = lib().spectre_prefix_readout_workspace_bytes(ctypes.byref(self.c), mode, io)
        self._ws, wsp, wsn = _workspace(need, g.device, self._ws)
        _check(lib().spectre_prefix_readout(ctypes.byref(self.c), _ptr(g, "g"), mode, _ptr(out, "out"), io, wsp, wsn,
                                            _stream(stream)))
        return out

    def step(self, v_t, q_t, P, out=None, stream=None):
        io = _dtype_code(v_t)
        if out is None:
            out = torch.empty((self.B, 1, self.H, self.d), dtype=v_t.dtype, device=v_t.device)
        need = lib().spectre_prefix_step_workspace_bytes(ctypes.byref(self.c), ctypes.byref(P.c))
        self._ws, wsp, wsn = _workspace(need, v_t.device, self._ws)
        _check(lib().spectre_prefix_step(ctypes.byref(self.c), _ptr(v_t, "v_t"), _ptr(q_t, "q_t"), ctypes.byref(P.c),
                                         _ptr(out, "out"), io, wsp, wsn, _stream(stream)))
        return out


def _rows(t, name, dtype, T=None, heads=None):
    """(address, elements from token to token) of rows [T, heads, d]: heads adjacent, tokens any distance apart."""
    if not t.is_cuda or t.dim() != 3:
        raise ValueError(f"{name} must be a device tensor [T, heads, d]")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, not {dtype}")
    n, h, d = t.shape
    if (T is not None and n != T) or (heads is not None and h != heads):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not [{T}, {heads}, d]")
    st, sh, sc = t.stride()
    if (sc != 1 and d > 1) or (sh != d and h > 1):
        raise ValueError(f"{name} must have its heads' channels adjacent")
    return t.data_ptr(), st if n > 1 else h * d


def _ints(t, name, n=None):
    if t.dtype != torch.int32:
        raise TypeError(f"{name} must be int32")
    if t.dim() != 1 or (n is not None and t.numel() != n):
        raise ValueError(f"{name} must be one-dimensional" + ("" if n is None else f" of {n} entries"))
    return _ptr(t, name)


def _new(shape, dtype, device, stream):
    """A tensor that work on `stream` (None: the current one) writes: its memory comes from that stream's blocks."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _like(t, stream):
    """The same with the shape and type of t, contiguous (half a microsecond less than by shape, type and device)."""
    if stream is None:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    with torch.cuda.stream(stream):
        return torch.empty_like(t, memory_format=torch.contiguous_format)


def _now(stream):
    """Raw handle of `stream` or the current one, for the calls that take tensors (so that the device is there): a serving step makes several."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if stream is None else stream.cuda_stream


def _capturing(stream):
    """Whether work on `stream` (None: the current one) is being captured into a graph."""
    if stream is None:
        return torch._C._cuda_isCurrentStreamCapturing()
    with torch.cuda.stream(stream):
        return torch._C._cuda_isCurrentStreamCapturing()


_kv_prepared = set()


def _kv_prepare():
    dev = torch.cuda.current_device()
    if dev not in _kv_prepared:
        _check(lib().spectre_kv_prepare())
        _kv_prepared.add(dev)


class Rope:
    """Angles by which a head's channels are turned: position * inv_freq[i] for pair i.  inv_freq: float64 [rot / 2] (any rule a model has for
    it), or use Rope.of for theta^(-2 i / rot).  axes: for tokens with several positions (time, height, width), the axis of each pair, integers
    [rot / 2] from 0 on; positions are then int32 [axes, T], with a row for each axis up to the largest that a pair has; rows behind it have no part."""

    MAX_AXES = 8

    def __init__(self, inv_freq, interleaved=False, device="cuda", axes=None):
        self.inv_freq = torch.as_tensor(inv_freq, dtype=torch.float64).to(device).contiguous()
        if self.inv_freq.dim() != 1:
            raise ValueError("inv_freq must be one-dimensional")
        self.rot, self.interleaved, self.axes, self.axis = 2 * self.inv_freq.numel(), bool(interleaved), 1, None
        if axes is not None:
            axis = torch.as_tensor(axes)
            if axis.is_floating_point() or axis.is_complex() or axis.dtype == torch.bool or tuple(axis.shape) != tuple(self.inv_freq.shape):
                raise ValueError("axes must be an integer for each of inv_freq")
            if axis.numel():
                if int(axis.min()) < 0 or int(axis.max()) >= self.MAX_AXES:
                    raise ValueError(f"axes must be between 0 and {self.MAX_AXES - 1}")
                self.axes = int(axis.max()) + 1
                self.axis = axis.to(device=device, dtype=torch.int32).contiguous()

    @classmethod
    def of(cls, rot, theta=10000.0, interleaved=False, device="cuda", axes=None):
        return cls(theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot), interleaved, device, axes)


def _heads(d, rope, wq, wk, eps):
    """The C parameters; rope None: no rotation, wq and wk None: no norm."""
    wq, wk = _vector(wq, "wq", d), _vector(wk, "wk", d)
    if rope is None:
        return HeadsC(d, 0, 0, eps, None, wq, wk, 1, None)
    if not rope.inv_freq.is_cuda:
        raise ValueError("rope must be on the device")
    return HeadsC(d, rope.rot, rope.interleaved, eps, rope.inv_freq.data_ptr(), wq, wk, rope.axes, None if rope.axis is None else rope.axis.data_ptr())


def _vector(w, name, d):
    """Address of weights float32 [d], None of none."""
    if w is None:
        return None
    if w.dtype != torch.float32 or w.shape != (d,):
        raise ValueError(f"{name} must be float32 [{d}]")
    return _ptr(w, name)


def _positions(positions, rope, T):
    """Address of the tokens' positions: int32 [T], or [axes, T]."""
    axes = rope.axes if rope else 1
    if positions is None:
        if axes > 1:
            raise ValueError(f"positions [{axes}, {T}] have to be given for a rotation by several axes")
        return None
    if positions.dim() == 1 and axes == 1:
        return _ints(positions, "positions", T)
    if positions.dtype != torch.int32:
        raise TypeError("positions must be int32")
    # rows of axes that no pair goes by lie behind those that are read
    if positions.dim() != 2 or positions.shape[1] != T or not axes <= positions.shape[0] <= Rope.MAX_AXES:
        raise ValueError(f"positions must have shape [{axes}, {T}]")
    return _ptr(positions, "positions")


def qk_norm_rotate(q, k, positions=None, rope=None, wq=None, wk=None, eps=1e-6, q_out=None, k_out=None, stream=None):
    """Norm of each query and key head and rotation by position in one pass (spectre_heads_forward).  q [T,H,d], k [T,Hkv,d] f32/bf16, tokens any
    16-byte multiple apart; positions int32 [T] (None: 0 .. T-1), [axes, T] for a rope of several axes; wq, wk float32 [d], both None: no norm.  Returns (q_out, k_out)."""
    T, H, d = q.shape
    Hkv = k.shape[1]
    io = _dtype_code(q)
    qa, qs = _rows(q, "q", q.dtype)
    ka, ks = _rows(k, "k", q.dtype, T)
    if k.shape[2] != d:
        raise ValueError("q and k differ in d")
    P = _heads(d, rope, wq, wk, eps)
    if q_out is None:
        q_out = _like(q, stream)
    else:
        _same(q_out, q, "q_out")
    if k_out is None:
        k_out = _like(k, stream)
    else:
        _same(k_out, k, "k_out")
    _check(lib().spectre_heads_forward(ctypes.byref(P), qa, qs, ka, ks, _positions(positions, rope, T), T, H, Hkv, io,
                                       _ptr(q_out, "q_out"), _ptr(k_out, "k_out"), _now(stream)))
    return q_out, k_out


def _same(t, like, name):
    if t.shape != like.shape or t.dtype != like.dtype:
        raise ValueError(f"{name} must be {like.dtype} {tuple(like.shape)}")


def qk_norm_rotate_backward(dq, dk, q, k, positions=None, rope=None, wq=None, wk=None, eps=1e-6, ws=None, stream=None):
    """Gradients of qk_norm_rotate (spectre_heads_backward) from those of its outputs and its inputs.
    Returns (gq, gk, gwq, gwk), the last two None without a norm."""
    T, H, d = q.shape
    Hkv = k.shape[1]
    io = _dtype_code(q)
    if tuple(k.shape) != (T, Hkv, d) or dq.shape != q.shape or dk.shape != k.shape:
        raise ValueError("dq and dk must have the shapes of q [T,H,d] and k [T,Hkv,d]")
    P = _heads(d, rope, wq, wk, eps)
    rows = [_rows(t, name, q.dtype) for t, name in ((dq, "dq"), (dk, "dk"), (q, "q"), (k, "k"))]
    gq, gk = _like(q, stream), _like(k, stream)
    gw, wsp, wsn = (None, None), None, 0
    if wq is not None and wk is not None:                                 # one of them alone is refused by the library
        gw = _like(wq, stream), _like(wk, stream)
        if ws is None:
            wsn = lib().spectre_heads_backward_workspace_bytes(T, d)
            ws = _new((wsn,), torch.uint8, q.device, stream)          # the allocator's memory is aligned
            wsp = ws.data_ptr()
        else:
            wsp, wsn = _given(ws)
    _check(lib().spectre_heads_backward(ctypes.byref(P), *rows[0], *rows[1], *rows[2], *rows[3],
                                        _positions(positions, rope, T), T, H, Hkv, io, gq.data_ptr(), gk.data_ptr(),
                                        None if gw[0] is None else gw[0].data_ptr(), None if gw[1] is None else gw[1].data_ptr(), wsp, wsn,
                                        _now(stream)))
    return gq, gk, gw[0], gw[1]


def _matrix(t, name, T, D, dtype):
    """(address, elements from row to row) of rows [T, D] whose channels are adjacent."""
    if not t.is_cuda or t.shape != (T, D):
        raise ValueError(f"{name} must be a device tensor [{T}, {D}]")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, not {dtype}")
    st, sc = t.stride()
    if sc != 1 and D > 1:
        raise ValueError(f"{name} must have adjacent channels")
    return t.data_ptr(), st if T > 1 else D


NORM_GROUP, NORM_MOST_BYTES = 128, 32768          # channels of a scale; the widest row


def add_norm(x, weight=None, delta=None, eps=1e-6, dtype=None, sum_out=None, out=None, scales=None, stream=None):
    """A residual's addition and the root-mean-square norm of the sum in one pass (spectre_norm_forward).  x, delta [T, D] f32/bf16, rows any 16-byte multiple
    apart; weight float32 [D] (None: ones); given outputs overlap no input.  Returns (sum, y), the sum in x's dtype (x itself without delta), y in x's dtype, or with dtype=torch.float8_e4m3fn
    (sum, codes, scales): a float32 scale for each 128 channels, scales [T, D / 128], and what is meant is code * scale."""
    T, D = x.shape
    io, kind, coded = _dtype_code(x), x.dtype, dtype == torch.float8_e4m3fn
    if dtype is not None and not coded and dtype != kind:
        raise TypeError(f"the norm of {kind} rows is {kind} or float8_e4m3fn, not {dtype}")
    xa, xs = _matrix(x, "x", T, D, kind)
    da, ds = (None, 0) if delta is None else _matrix(delta, "delta", T, D, kind)
    if delta is None:
        if sum_out is not None:
            raise ValueError("without delta there is no sum")
    elif sum_out is None:
        sum_out = _like(x, stream)
    else:
        _same(sum_out, x, "sum_out")
    if coded:
        if D % NORM_GROUP:
            raise ValueError(f"rows of 8 bits have a multiple of {NORM_GROUP} channels")
        if out is None:
            out = _new((T, D), dtype, x.device, stream)
        if scales is None:
            scales = _new((T, D // NORM_GROUP), torch.float32, x.device, stream)
        elif scales.dtype != torch.float32 or tuple(scales.shape) != (T, D // NORM_GROUP):
            raise ValueError(f"scales must be float32 [{T}, {D // NORM_GROUP}]")
        if out.dtype != dtype or tuple(out.shape) != (T, D):
            raise ValueError(f"out must be {dtype} [{T}, {D}]")
    elif scales is not None:
        raise ValueError("scales are of 8 bits' rows")
    elif out is None:
        out = _like(x, stream)
    else:
        _same(out, x, "out")
    _check(lib().spectre_norm_forward(xa, xs, da, ds, _vector(weight, "weight", D), T, D, eps, io, None if delta is None else _ptr(sum_out, "sum_out"), _ptr(out, "out"),
                                      E4M3 if coded else io, _ptr(scales, "scales") if coded else None, _now(stream)))
    total = x if delta is None else sum_out
    return (total, out, scales) if coded else (total, out)


def add_norm_backward(dy, total, weight=None, dsum=None, eps=1e-6, ws=None, stream=None):
    """Gradients of add_norm (spectre_norm_backward): dy of its y (in the rows' dtype, of 8 bits' rows as if they had not been rounded), total: the sum it returned,
    dsum: the gradient of that sum where it goes on as a residual (None: nothing comes from there).  Returns (gx, gw): gx is the gradient of x and of delta, gw float32
    [D], None without a weight."""
    T, D = total.shape
    io, kind = _dtype_code(total), total.dtype
    ta, ts = _matrix(total, "total", T, D, kind)
    ya, ys = _matrix(dy, "dy", T, D, kind)
    da, ds = (None, 0) if dsum is None else _matrix(dsum, "dsum", T, D, kind)
    w = _vector(weight, "weight", D)
    gx, gw, wsp, wsn = _like(total, stream), None, None, 0
    if weight is not None:
        gw = _like(weight, stream)
        if ws is None:
            wsn = lib().spectre_norm_backward_workspace_bytes(T, D, io)
            if wsn:
                ws = _new((wsn,), torch.uint8, total.device, stream)  # the allocator's memory is aligned
                wsp = ws.data_ptr()
        else:
            wsp, wsn = _given(ws)
    _check(lib().spectre_norm_backward(ya, ys, ta, ts, da, ds, w, T, D, eps, io, _ptr(gx, "gx"), None if gw is None else _ptr(gw, "gw"), wsp, wsn, _now(stream)))
    return gx, gw


class KvPages:
    """Keys and values of attention layers in pages, with their bookkeeping on the device (spectre_kv; layout and rules in spectre.h).

    KvPages.empty(...) allocates an empty pool; the constructor takes tensors that exist:
    k_pages [layers, pages, Hkv, d/E, page, E], v_pages [layers, pages, Hkv, page/E, d, E] (E = 8 bf16, 4 f32 or 16 float8_e4m3fn elements),
    book int32 [8 + seqs + pages + seqs * max_pages]; with pages of float8_e4m3fn, whose rows are bf16, also scales float32
    [layers, pages, Hkv, page/16, 2], powers of two: of the keys and of the values of each 16 tokens of a head (what is stored is code * scale)."""

    NO_PAGES, TOO_LONG, BAD_ARGUMENT, NOT_EMPTY, SHARED = 1, 2, 4, 8, 16          # bits of the status

    BLOCK = 16                          # tokens of a page of 8 bits that share a scale

    def __init__(self, k_pages, v_pages, book, seqs, max_pages, scales=None):
        io = E4M3 if k_pages.dtype == torch.float8_e4m3fn else _dtype_code(k_pages)
        E = 16 // k_pages.element_size()
        if k_pages.dim() != 6 or k_pages.shape[5] != E:
            raise ValueError(f"k_pages must be [layers, pages, Hkv, d/{E}, page, {E}]")
        layers, pages, Hkv, groups, page, _ = k_pages.shape
        d = groups * E
        if tuple(v_pages.shape) != (layers, pages, Hkv, page // E, d, E) or v_pages.dtype != k_pages.dtype:
            raise ValueError(f"v_pages must be {k_pages.dtype} [layers, pages, Hkv, page/{E}, d, {E}]")
        if (scales is not None) != (io == E4M3):
            raise ValueError("pages of float8_e4m3fn have scales, others none")
        if scales is not None and (scales.dtype != torch.float32 or tuple(scales.shape) != (layers, pages, Hkv, page // self.BLOCK, 2)):
            raise ValueError(f"scales must be float32 [layers, pages, Hkv, page/{self.BLOCK}, 2]")
        if book.numel() != 8 + seqs + pages + seqs * max_pages:
            raise ValueError("book must have 8 + seqs + pages + seqs * max_pages entries")
        self.layers, self.pages, self.Hkv, self.d, self.page, self.seqs, self.max_pages = layers, pages, Hkv, d, page, seqs, max_pages
        self.dtype, self.k_pages, self.v_pages, self.book, self.scales = k_pages.dtype, k_pages, v_pages, book, scales
        self.rows = torch.bfloat16 if io == E4M3 else self.dtype               # type of the rows that calls take
        self.c = KvC(layers, pages, Hkv, d, page, seqs, max_pages, io, _ptr(k_pages, "k_pages"), _ptr(v_pages, "v_pages"), _ints(book, "book"),
                     None if scales is None else _ptr(scales, "scales"))
        self._ref = ctypes.byref(self.c)
        if lib().spectre_kv_bytes(self._ref, 0) == 0:
            raise SpectreError(EUNSUPPORTED, lib().spectre_last_error().decode())
        _kv_prepare()
        self._ws = {}

    @classmethod
    def empty(cls, layers, pages, Hkv, d, page, seqs, max_pages, dtype=torch.bfloat16, device="cuda"):
        codes = {torch.bfloat16: BF16, torch.float8_e4m3fn: E4M3}
        c = KvC(layers, pages, Hkv, d, page, seqs, max_pages, codes.get(dtype, F32), None, None, None, None)
        n = lib().spectre_kv_bytes(ctypes.byref(c), 0)
        if n == 0:
            raise SpectreError(EUNSUPPORTED, lib().spectre_last_error().decode())
        E = 16 // dtype.itemsize
        scales = torch.ones((layers, pages, Hkv, page // cls.BLOCK, 2), device=device) if dtype == torch.float8_e4m3fn else None
        k = torch.zeros((layers, pages, Hkv, d // E, page, E), dtype=dtype, device=device)
        v = torch.zeros((layers, pages, Hkv, page // E, d, E), dtype=dtype, device=device)
        book = torch.empty(8 + seqs + pages + seqs * max_pages, dtype=torch.int32, device=device)
        pool = cls(k, v, book, seqs, max_pages, scales)
        pool.reset()
        return pool

    def reset(self, stream=None):
        """No sequence has a token, no page a user."""
        _check(lib().spectre_kv_init(self._ref, _now(stream)))

    # views of the bookkeeping, on the device
    @property
    def status(self):
        return self.book[:8]

    @property
    def lens(self):
        return self.book[8:8 + self.seqs]

    @property
    def refs(self):
        return self.book[8 + self.seqs:8 + self.seqs + self.pages]

    @property
    def table(self):
        return self.book[8 + self.seqs + self.pages:].view(self.seqs, self.max_pages)

    def _scratch(self, kind, stream, now, need=0):
        """(address, bytes) of the pool's workspace, kept between calls (one for the attention, one for the pages: a pool works on one stream at a time);
        now: the stream's handle.  Captured calls have memory of their own instead, which lives as long as their graph: this one is replaced as soon as a call needs more."""
        own, raw, at, have = self._ws.get(kind, (None, 0, None, 0))
        if have < need:
            own = _new((need + 256,), torch.uint8, self.book.device, stream)
            at, have = _given(own)
            self._ws[kind] = own, now, at, have
        elif now != raw and own is not None:   # the allocator must not give its memory away while another stream works with it
            own.record_stream(torch.cuda.current_stream() if stream is None else stream)
        return at, have

    def _fresh(self, need, stream):
        """Workspace of one captured call.  Its caller holds it until the call has been captured; the graph keeps the memory from then on."""
        return _new((need + 256,), torch.uint8, self.book.device, stream)

    def _pages_call(self, call, lists, n, ws, stream):
        """reserve, fork or compact with their lists, a workspace (of a list of n) and the stream."""
        now = _now(stream)
        if ws is None:
            need = lib().spectre_kv_workspace_bytes(self._ref, n)
            if _capturing(stream):
                ws = self._fresh(need, stream)
        at, have = self._scratch("pages", stream, now, need) if ws is None else _given(ws)
        _check(call(self._ref, *lists, at, have, now))

    def reserve(self, seqs, add, ws=None, stream=None):
        """Sequence seqs[i] grows by add[i] tokens (int32 on the device); room that is missing is reported in `status`, and then nothing changes, nor does
        append() write anything until status[0] has been cleared."""
        n = seqs.numel()
        self._pages_call(lib().spectre_kv_reserve, (_ints(seqs, "seqs"), _ints(add, "add", n), n), n, ws, stream)

    def fork(self, src, dst, ws=None, stream=None):
        """The empty sequences dst[i] become what src[i] are: full pages shared, the last one copied."""
        n = src.numel()
        self._pages_call(lib().spectre_kv_fork, (_ints(src, "src"), _ints(dst, "dst", n), n), n, ws, stream)

    def free(self, seqs, stream=None):
        """The sequences end; pages that nobody else uses are free."""
        _check(lib().spectre_kv_free(self._ref, _ints(seqs, "seqs"), seqs.numel(), _now(stream)))

    def compact(self, ws=None, stream=None):
        """Pages in use move to the front of the pool; status[2] = how many there are."""
        self._pages_call(lib().spectre_kv_compact, (), 0, ws, stream)

    def copy(self, src, dst, stream=None):
        """Contents of page src[i] of every layer to page dst[i]."""
        n = src.numel()
        _check(lib().spectre_kv_copy(self._ref, _ints(src, "src"), _ints(dst, "dst", n), n, _now(stream)))

    def append(self, layer, q, k, v, start, seqs=None, rope=None, wq=None, wk=None, eps=1e-6, q_out=None, stream=None, positions=None):
        """Norm and rotation of the new tokens' heads; keys and values go into the pages of `layer`, queries are returned.  q [T,H,d], k, v [T,Hkv,d] of the
        pool's dtype (bf16 for pages of 8 bits); start int32 [B+1]: first token of each sequence; seqs int32 [B]: their rows of the table (None: 0 .. B-1).  The new tokens are
        the last ones of their sequences: reserve() comes first, once for all layers.  While NO_PAGES, TOO_LONG or BAD_ARGUMENT stands in status[0] nothing is
        written, nor is anything into a page that several sequences use (SHARED).  positions: what the rotation goes by, int32 [T] or [axes, T] (None: the
        places in the sequences, of a rope of one axis); where keys are stored and what a query sees goes by the order of the tokens."""
        T, H, d = q.shape
        B = start.numel() - 1
        qa, qs = _rows(q, "q", self.rows)
        ka, ks = _rows(k, "k", self.rows, T, self.Hkv)
        va, vs = _rows(v, "v", self.rows, T, self.Hkv)
        if d != self.d or k.shape[2] != d or v.shape[2] != d:
            raise ValueError(f"q, k and v must have d = {self.d}")
        P = _heads(d, rope, wq, wk, eps)
        if q_out is None:
            q_out = _like(q, stream)
        else:
            _same(q_out, q, "q_out")
        _check(lib().spectre_kv_append_at(self._ref, layer, ctypes.byref(P), qa, qs, ka, ks, va, vs, _positions(positions, rope, T), _ints(start, "start"),
                                          None if seqs is None else _ints(seqs, "seqs", B), B, T, H, _ptr(q_out, "q_out"), _now(stream)))
        return q_out

    def attend_workspace_bytes(self, B, T, H, max_new, max_len=None, window=0):
        return int(lib().spectre_kv_attend_workspace_bytes(self._ref, B, T, H, max_new, max_len or self.max_pages * self.page, window))

    def attend(self, layer, q, start, seqs=None, max_new=None, max_len=None, scale=None, window=0, out=None, lse=None, want_lse=False, ws=None,
               stream=None):
        """Attention of the new tokens (append has written their keys and values) over their sequences' pages (spectre_kv_attend).
        max_new, max_len: bounds of the sequences' new tokens and lengths (None: T, and the table's width), which the launch, its workspace and with them its time are
        sized by: give them wherever the program knows them (a batch of single tokens without max_new=1 runs as one of chunks of T); scale None: d^-1/2; window > 0: each
        query sees that many keys, its own the last.  Returns out [T,H,d], with want_lse or a tensor `lse` also lse float32 [T,H]."""
        T, H, d = q.shape
        B = start.numel() - 1
        qa, qs = _rows(q, "q", self.rows)
        if d != self.d:
            raise ValueError(f"q must have d = {self.d}")
        if max_new is None:
            max_new = max(T, 1)
        if max_len is None:
            max_len = self.max_pages * self.page
        if out is None:
            out = _like(q, stream)
        else:
            _same(out, q, "out")
        if lse is None:
            if want_lse:
                lse = _new((T, H), torch.float32, q.device, stream)
        elif lse.dtype != torch.float32 or tuple(lse.shape) != (T, H):
            raise ValueError("lse must be float32 [T, H]")
        args = (self._ref, layer, qa, qs, _ints(start, "start"), None if seqs is None else _ints(seqs, "seqs", B), B, T, H, max_new, max_len,
                1.0 / d ** 0.5 if scale is None else scale, window, _ptr(out, "out"), None if lse is None else _ptr(lse, "lse"))
        now = _now(stream)
        if ws is None and _capturing(stream):
            ws = self._fresh(lib().spectre_kv_attend_workspace_bytes(self._ref, B, T, H, max_new, max_len, window), stream)
        at, have = _given(ws) if ws is not None else self._scratch("attend", stream, now)
        rc = lib().spectre_kv_attend(*args, at, have, now)
        if rc == EWORKSPACE and ws is None:    # the library checks the size; asking for it first is a call of its own
            at, have = self._scratch("attend", stream, now, lib().spectre_kv_attend_workspace_bytes(self._ref, B, T, H, max_new, max_len, window))
            rc = lib().spectre_kv_attend(*args, at, have, now)
        _check(rc)
        return (out, lse) if lse is not None else out
