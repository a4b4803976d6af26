"""ctypes binding of libsparsek.so.  Function names mirror include/sparsek.h."""
import ctypes as C
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsparsek.so")
_lib = None

F32, BF16, I8, E4M3, E2M1 = 0, 1, 2, 3, 4
BLOCK_TOKENS = 64


class SparsekCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "H", "Gu", "n", "d", "k", "w", "dtype", "gate_mode")] + [
        ("softmax_scale", C.c_float)
    ]


class SparsekScoresCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "n", "D", "dtype", "norm")] + [("slope", C.c_float), ("norm_eps", C.c_float)]


class SparsekChunkCfg(C.Structure):
    _fields_ = [
        (n, C.c_int32) for n in ("B", "H", "Gu", "d", "k", "w", "cand_cap", "chunk_max", "dtype", "gate_mode")
    ] + [("softmax_scale", C.c_float)]


class SparsekDecodeCfg(C.Structure):
    _fields_ = [
        (n, C.c_int32) for n in ("B", "H", "Gu", "d", "k", "w", "cand_cap", "dtype", "gate_mode")
    ] + [("softmax_scale", C.c_float)]


class SparsekBlockCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "H", "Hkv", "n", "d", "top", "dtype")] + [("softmax_scale", C.c_float)]


class SparsekCache8Cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "H", "Hkv", "d", "cap", "pages", "format", "dtype")] + [("softmax_scale", C.c_float)]


class SparsekRopeStrides(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("batch", "token", "head")]


class SparsekRopeCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "H", "Hkv", "n", "d", "rot", "axes", "interleaved", "norm", "dtype")] + [
        ("eps", C.c_float)] + [(n, SparsekRopeStrides) for n in ("q", "k", "dq", "dk")]


_CACHE8_TENSORS = ("k8", "v8", "ks", "vs", "km", "kms", "kt", "vt", "table", "mass")


class SparsekCache8(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _CACHE8_TENSORS]


_CACHE4_TENSORS = ("k4", "v4", "ke", "ve") + _CACHE8_TENSORS[2:]


class SparsekCache4(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in _CACHE4_TENSORS]


def lib_path():
    return _LIB_PATH


def lib():
    """The loaded C-ABI library.  Raises if it has not been built (no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                "libsparsek.so is missing: build it with `python -m paper_2406_16747_amd.build` "
                "(there is no CPU fallback)"
            )
        L = C.CDLL(_LIB_PATH)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        cfgp, dcfgp = C.POINTER(SparsekCfg), C.POINTER(SparsekDecodeCfg)
        L.sparsek_strerror.restype = C.c_char_p
        L.sparsek_strerror.argtypes = [C.c_int]
        for name in ("sparsek_mask_workspace_bytes", "sparsek_attn_fwd_workspace_bytes",
                     "sparsek_mask_bwd_workspace_bytes", "sparsek_attn_bwd_workspace_bytes"):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = [cfgp]
        L.sparsek_mask.argtypes = [cfgp, vp, vp, vp, vp, sz, vp]
        L.sparsek_mask_status.argtypes = [cfgp, vp, sz, vp, vp]
        L.sparsek_mask_status.restype = C.c_int
        L.sparsek_mask_static.argtypes = [cfgp, vp, vp, vp, vp]
        L.sparsek_mask_static.restype = C.c_int
        L.sparsek_materialize.argtypes = [cfgp, vp, vp, vp, i32, i32, vp, vp, vp]
        L.sparsek_attn_fwd.argtypes = [cfgp] + [vp] * 8 + [vp, sz, vp]
        L.sparsek_mask_bwd.argtypes = [cfgp] + [vp] * 10 + [vp, sz, vp]
        L.sparsek_attn_bwd.argtypes = [cfgp] + [vp] * 12 + [vp, sz, vp]
        L.sparsek_attn_bwd.restype = C.c_int
        L.sparsek_bwd.argtypes = [cfgp] + [vp] * 13 + [vp, sz, vp]
        L.sparsek_bwd.restype = C.c_int
        L.sparsek_bwd_workspace_bytes.restype = sz
        L.sparsek_bwd_workspace_bytes.argtypes = [cfgp]
        scfgp = C.POINTER(SparsekScoresCfg)
        L.sparsek_scores_workspace_bytes.restype = sz
        L.sparsek_scores_workspace_bytes.argtypes = [scfgp]
        L.sparsek_scores.argtypes = [scfgp, vp, vp, vp, vp, sz, vp]
        L.sparsek_scores.restype = C.c_int
        ccfgp = C.POINTER(SparsekChunkCfg)
        for name in ("sparsek_chunk_state_bytes", "sparsek_chunk_workspace_bytes", "sparsek_chunk_bwd_workspace_bytes"):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = [ccfgp]
        L.sparsek_chunk_init.argtypes = [ccfgp, vp, sz, vp]
        L.sparsek_chunk_prefill.argtypes = [ccfgp, vp, sz, i32] + [vp] * 5 + [vp, sz, vp]
        L.sparsek_chunk_status.argtypes = [ccfgp, vp, vp, vp, vp]
        L.sparsek_chunk_bwd.argtypes = [ccfgp, i32, vp, vp, vp, vp, sz, vp, vp, vp, vp, vp, sz, vp]
        L.sparsek_chunk_bwd.restype = C.c_int
        L.sparsek_chunk_to_decode.argtypes = [ccfgp, vp, sz, C.c_int64, vp, sz, dcfgp, vp, sz, vp]
        for name in ("sparsek_chunk_init", "sparsek_chunk_prefill", "sparsek_chunk_status", "sparsek_chunk_to_decode"):
            getattr(L, name).restype = C.c_int
        L.sparsek_decode_state_bytes.restype = sz
        L.sparsek_decode_state_bytes.argtypes = [dcfgp]
        L.sparsek_decode_init.argtypes = [dcfgp, vp, sz, vp]
        L.sparsek_decode_load.argtypes = [dcfgp, vp, sz, i32] + [vp] * 5 + [vp]
        L.sparsek_decode_step.argtypes = [dcfgp, vp] + [vp] * 5 + [vp]
        L.sparsek_decode_status.argtypes = [dcfgp, vp, vp, vp]
        for name in ("sparsek_mask", "sparsek_materialize", "sparsek_attn_fwd", "sparsek_mask_bwd",
                     "sparsek_decode_init", "sparsek_decode_load", "sparsek_decode_step",
                     "sparsek_decode_status"):
            getattr(L, name).restype = C.c_int
        bcfgp, c8cfgp, c8p = C.POINTER(SparsekBlockCfg), C.POINTER(SparsekCache8Cfg), C.POINTER(SparsekCache8)
        for name in ("sparsek_block_select_workspace_bytes", "sparsek_block_attn_fwd_workspace_bytes",
                     "sparsek_block_attn_bwd_workspace_bytes"):
            getattr(L, name).restype = sz
            getattr(L, name).argtypes = [bcfgp]
        L.sparsek_block_select.argtypes = [bcfgp, vp, vp, vp, vp, sz, vp]
        L.sparsek_block_attn_fwd.argtypes = [bcfgp] + [vp] * 7 + [vp, sz, vp]
        L.sparsek_block_attn_bwd.argtypes = [bcfgp] + [vp] * 10 + [vp, sz, vp]
        for cache, cp in (("sparsek_cache8_", c8p), ("sparsek_cache4_", C.POINTER(SparsekCache4))):
            for name, types in (("append", [vp, vp, i32, vp, vp]), ("select", [vp, vp, i32, vp]), ("evict", [vp, i32, i32, i32, vp, vp, vp]),
                                ("attn", [vp, vp, vp, i32, i32, vp, vp, vp, sz]), ("read", [vp, i32, i32, vp, vp])):
                if name == "read" and cp is c8p:
                    continue
                getattr(L, cache + name).argtypes = [c8cfgp, cp] + types + [vp]
                getattr(L, cache + name).restype = C.c_int
            getattr(L, cache + "attn_workspace_bytes").restype = sz
            getattr(L, cache + "attn_workspace_bytes").argtypes = [c8cfgp, i32]
        for name in ("sparsek_block_select", "sparsek_block_attn_fwd", "sparsek_block_attn_bwd"):
            getattr(L, name).restype = C.c_int
        rcfgp = C.POINTER(SparsekRopeCfg)
        L.sparsek_rope_bwd_workspace_bytes.restype = sz
        L.sparsek_rope_bwd_workspace_bytes.argtypes = [rcfgp]
        L.sparsek_rope_fwd.argtypes = [rcfgp] + [vp] * 9 + [vp]
        L.sparsek_rope_bwd.argtypes = [rcfgp] + [vp] * 13 + [vp, sz, vp]
        L.sparsek_rope_fwd.restype = L.sparsek_rope_bwd.restype = C.c_int
        _lib = L
    return _lib


def check(rc):
    if rc != 0:
        raise RuntimeError("libsparsek: %s (%d)" % (lib().sparsek_strerror(rc).decode(), rc))


# Host time per call matters where the kernels take a few microseconds: configurations (with their workspace sizes) are
# kept, pointers are passed as plain integers, and the stream is asked for without building a Stream object.
torch = None
_raw_stream = None
_here = None      # the current device; the stream of a device, as an integer
_CFG_KEPT = 256   # configurations kept per kind
_cfgs = {}


def _torch():
    global torch, _raw_stream, _here
    if torch is None:
        import torch as t

        get, dev = getattr(t._C, "_cuda_getCurrentRawStream", None), getattr(t._C, "_cuda_getDevice", None)
        _raw_stream = (lambda: get(dev())) if get and dev else (lambda: t.cuda.current_stream().cuda_stream)
        if get and dev:
            _here = dev, get
        else:
            _here = t.cuda.current_device, lambda device: t.cuda.current_stream(device).cuda_stream
        torch = t
    return torch


def _stream():
    return (_raw_stream or (_torch() and _raw_stream))()


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _dtype_code(t):
    _torch()
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return F32
    raise TypeError("q,k,v must be float32 or bfloat16, got %s" % t.dtype)


def _need(t, dtype, name):
    if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor on the GPU" % (name, dtype))


def _ws(nbytes, device):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _kept(kind, key, make):
    """(reference to pass, configuration, {query: bytes}) of a configuration, made once."""
    d = _cfgs.get(kind)
    if d is None:
        d = _cfgs.setdefault(kind, {})
    got = d.get(key)
    if got is None:
        cfg = make(*key)
        got = (C.byref(cfg), cfg, {})
        if len(d) >= _CFG_KEPT:
            d.clear()
        d[key] = got
    return got


def _bytes(kept, query):
    n = kept[2].get(query)
    if n is None:
        n = kept[2][query] = max(int(getattr(lib(), query)(kept[0])), 256)
    return n


def _make_mask_cfg(B, Gu, n, k):
    return SparsekCfg(B=B, H=Gu, Gu=Gu, n=n, d=64, k=k, w=1, dtype=F32, gate_mode=0, softmax_scale=1.0)


def _mask_kept(u, k):
    B, Gu, n = u.shape
    return _kept("mask", (B, Gu, n, int(k)), _make_mask_cfg)


def sparsek_mask(u, k, ws=None):
    """u [B,Gu,n] fp32 -> (tau [B,Gu,n] fp32, death [B,Gu,n] int32)."""
    torch, L = _torch(), lib()
    _need(u, torch.float32, "u")
    cfg = _mask_kept(u, k)
    tau = torch.empty_like(u)
    death = torch.empty_like(u, dtype=torch.int32)
    if ws is None:
        nbytes = _bytes(cfg, "sparsek_mask_workspace_bytes")
        ws = torch.empty(nbytes, dtype=torch.uint8, device=u.device)
    else:
        nbytes = ws.numel()
    rc = L.sparsek_mask(cfg[0], u.data_ptr(), tau.data_ptr(), death.data_ptr(), ws.data_ptr(), nbytes, _raw_stream())
    if rc:
        check(rc)
    return tau, death


def sparsek_mask_static(u, k, tau=None, death=None):
    """sparsek_mask without a workspace (the library's built-in scratch array); tau, death may be preallocated."""
    torch = _torch()
    _need(u, torch.float32, "u")
    cfg = _mask_kept(u, k)
    if tau is None:
        tau = torch.empty_like(u)
    if death is None:
        death = torch.empty(u.shape, dtype=torch.int32, device=u.device)
    _need(tau, torch.float32, "tau")
    _need(death, torch.int32, "death")
    check(lib().sparsek_mask_static(cfg[0], _ptr(u), _ptr(tau), _ptr(death), _stream()))
    return tau, death


def sparsek_mask_workspace(u, k):
    """A workspace for sparsek_mask(u, k, ws=...), to be read back with sparsek_mask_status."""
    _torch()
    return _ws(lib().sparsek_mask_workspace_bytes(_mask_kept(u, k)[0]), u.device)


def sparsek_mask_status(u, k, ws):
    """Status word of the last sparsek_mask(u, k, ws=ws) call (0 = every threshold solve converged).  Synchronises."""
    flag = C.c_int32(-1)
    _torch()
    check(lib().sparsek_mask_status(_mask_kept(u, k)[0], _ptr(ws), ws.numel(), C.byref(flag), _stream()))
    return int(flag.value)


def sparsek_materialize(u, tau, death, k, t_begin, t_end, with_gate=True):
    """Explicit top-k lists of prefixes [t_begin, t_end): idx, gate [B,Gu,nt,k]."""
    torch = _torch()
    B, Gu, n = u.shape
    cfg = SparsekCfg(B=B, H=Gu, Gu=Gu, n=n, d=64, k=int(k), w=1, dtype=F32, gate_mode=0, softmax_scale=1.0)
    nt = t_end - t_begin
    idx = torch.full((B, Gu, nt, max(int(k), 0)), -1, dtype=torch.int32, device=u.device)
    gate = torch.zeros((B, Gu, nt, max(int(k), 0)), dtype=torch.float32, device=u.device) if with_gate else None
    if idx.numel() == 0:
        return idx, gate
    check(lib().sparsek_materialize(C.byref(cfg), _ptr(u), _ptr(tau), _ptr(death), int(t_begin), int(t_end),
                                    _ptr(idx), _ptr(gate), _stream()))
    return idx, gate


def _make_attn_cfg(B, H, Gu, n, d, k, w, dtype, gate_mode, scale):
    return SparsekCfg(B=B, H=H, Gu=Gu, n=n, d=d, k=k, w=w, dtype=dtype, gate_mode=gate_mode, softmax_scale=scale)


def _attn_kept(q, u, k, w, gate_mode, scale):
    B, H, n, d = q.shape
    return _kept("attn", (B, H, u.shape[1], n, d, int(k), int(w), _dtype_code(q), int(gate_mode), float(scale)),
                 _make_attn_cfg)


def _attn_cfg(q, u, k, w, gate_mode, scale):
    """A configuration of the caller's own, for the size queries of the C interface."""
    B, H, n, d = q.shape
    return _make_attn_cfg(B, H, u.shape[1], n, d, int(k), int(w), _dtype_code(q), int(gate_mode), float(scale))


def _attn_ws(cfg, query, ws, device):
    """(workspace, its size): the caller's, or a new one of the size the query says."""
    if ws is not None:
        return ws, ws.numel()
    n = _bytes(cfg, query)
    return torch.empty(n, dtype=torch.uint8, device=device), n


def sparsek_attn_fwd(q, k, v, u, tau, death, k_sel, w, gate_mode=0, scale=1.0, return_lse=True, ws=None):
    """q,k,v [B,H,n,d]; u,tau,death [B,Gu,n] -> o [B,H,n,d] (and lse [B,H,n] fp32)."""
    torch, L = _torch(), lib()
    cfg = _attn_kept(q, u, k_sel, w, gate_mode, scale)
    dt, f32 = q.dtype, torch.float32
    _need(q, dt, "q")
    _need(k, dt, "k")
    _need(v, dt, "v")
    _need(u, f32, "u")
    _need(tau, f32, "tau")
    _need(death, torch.int32, "death")
    o = torch.empty_like(q)
    lse = torch.empty(q.shape[:3], dtype=f32, device=q.device) if return_lse else None
    ws, nbytes = _attn_ws(cfg, "sparsek_attn_fwd_workspace_bytes", ws, q.device)
    rc = L.sparsek_attn_fwd(cfg[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), u.data_ptr(), tau.data_ptr(), death.data_ptr(),
                            o.data_ptr(), lse.data_ptr() if return_lse else None, ws.data_ptr(), nbytes, _raw_stream())
    if rc:
        check(rc)
    return (o, lse) if return_lse else o


def sparsek_mask_bwd(q, k, v, u, tau, death, o, lse, dO, k_sel, w, gate_mode=0, scale=1.0, ws=None):
    """du [B,Gu,n] fp32: gradient of sum(dO*O) w.r.t. the scores through the soft gates."""
    torch, L = _torch(), lib()
    cfg = _attn_kept(q, u, k_sel, w, gate_mode, scale)
    du = torch.empty_like(u)
    ws, nbytes = _attn_ws(cfg, "sparsek_mask_bwd_workspace_bytes", ws, q.device)
    check(L.sparsek_mask_bwd(cfg[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), u.data_ptr(), tau.data_ptr(),
                             death.data_ptr(), o.data_ptr(), lse.data_ptr(), dO.data_ptr(), du.data_ptr(), ws.data_ptr(),
                             nbytes, _raw_stream()))
    return du


def sparsek_attn_bwd(q, k, v, u, tau, death, o, lse, dO, k_sel, w, gate_mode=0, scale=1.0, ws=None):
    """dq, dk, dv [B,H,n,d]: gradients of sum(dO*O) with respect to q, k, v (gates held fixed)."""
    torch, L = _torch(), lib()
    cfg = _attn_kept(q, u, k_sel, w, gate_mode, scale)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws, nbytes = _attn_ws(cfg, "sparsek_attn_bwd_workspace_bytes", ws, q.device)
    check(L.sparsek_attn_bwd(cfg[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), u.data_ptr(), tau.data_ptr(),
                             death.data_ptr(), o.data_ptr(), lse.data_ptr(), dO.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                             dv.data_ptr(), ws.data_ptr(), nbytes, _raw_stream()))
    return dq, dk, dv


def sparsek_bwd(q, k, v, u, tau, death, o, lse, dO, k_sel, w, gate_mode=0, scale=1.0, ws=None):
    """The whole backward in one call: (dq, dk, dv, du)."""
    torch, L = _torch(), lib()
    cfg = _attn_kept(q, u, k_sel, w, gate_mode, scale)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    du = torch.empty_like(u)
    ws, nbytes = _attn_ws(cfg, "sparsek_bwd_workspace_bytes", ws, q.device)
    check(L.sparsek_bwd(cfg[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), u.data_ptr(), tau.data_ptr(), death.data_ptr(),
                        o.data_ptr(), lse.data_ptr(), dO.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                        du.data_ptr(), ws.data_ptr(), nbytes, _raw_stream()))
    return dq, dk, dv, du


def _make_scores_cfg(B, n, D, dtype, norm, slope, norm_eps):
    return SparsekScoresCfg(B=B, n=n, D=D, dtype=dtype, norm=norm, slope=slope, norm_eps=norm_eps)


def sparsek_scores(x, w, slope=0.0, norm=False, norm_eps=1e-5, ws=None):
    """u [B,n] fp32 from hidden states x [B,n,D] (bf16 or fp32) and the scorer w [D] fp32:
    x.w + position slope, optionally timestep-normalised."""
    torch, L = _torch(), lib()
    B, n, D = x.shape
    assert x.is_contiguous() and w.is_contiguous() and w.dtype == torch.float32 and w.numel() == D
    dt = BF16 if x.dtype == torch.bfloat16 else F32
    assert dt == BF16 or x.dtype == torch.float32
    cfg = _kept("scores", (B, n, D, dt, int(bool(norm)), float(slope), float(norm_eps)), _make_scores_cfg)
    u = torch.empty(B, n, dtype=torch.float32, device=x.device)
    ws, nbytes = _attn_ws(cfg, "sparsek_scores_workspace_bytes", ws, x.device)
    check(L.sparsek_scores(cfg[0], x.data_ptr(), w.data_ptr(), u.data_ptr(), ws.data_ptr(), nbytes, _raw_stream()))
    return u


class ChunkState:
    """Caller-owned state of the chunk-wise recurrent prefill: a config, the state buffer and scratch."""

    def __init__(self, B, H, Gu, d, k, w, dtype, chunk_max, gate_mode=0, scale=1.0, cand_cap=0, device="cuda"):
        torch = _torch()
        self.cfg = SparsekChunkCfg(B=B, H=H, Gu=Gu, d=d, k=int(k), w=int(w), cand_cap=int(cand_cap),
                                   chunk_max=int(chunk_max), dtype=dtype, gate_mode=int(gate_mode),
                                   softmax_scale=float(scale))
        nbytes = lib().sparsek_chunk_state_bytes(self.cfg)
        if nbytes == 0:
            raise ValueError("invalid chunk configuration")
        self.buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.ws = torch.empty(lib().sparsek_chunk_workspace_bytes(self.cfg), dtype=torch.uint8, device=device)
        check(lib().sparsek_chunk_init(self.cfg, _ptr(self.buf), self.buf.numel(), _stream()))


def sparsek_chunk_prefill(state, q, k, v, u):
    """Attention output [B,H,c,d] of one chunk; the state moves on to the end of the chunk."""
    torch = _torch()
    c = q.shape[2]
    o = torch.empty_like(q)
    check(lib().sparsek_chunk_prefill(state.cfg, _ptr(state.buf), state.buf.numel(), c, _ptr(q), _ptr(k),
                                      _ptr(v), _ptr(u), _ptr(o), _ptr(state.ws), state.ws.numel(), _stream()))
    return o


def sparsek_chunk_bwd(state, q, o, dO):
    """Gradients (dq, dk, dv [B,H,c,d], du [B,Gu,c]) of sum(dO * o) for the chunk that the last
    sparsek_chunk_prefill call on this state processed, the retained keys of earlier chunks held constant."""
    torch = _torch()
    c = q.shape[2]
    nbytes = lib().sparsek_chunk_bwd_workspace_bytes(state.cfg)
    if nbytes == 0:
        raise ValueError("sparsek_chunk_bwd: unsupported configuration (bf16 with d = 64 or 128 only)")
    if getattr(state, "bwd_ws", None) is None or state.bwd_ws.numel() < nbytes:
        state.bwd_ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    du = torch.empty((state.cfg.B, state.cfg.Gu, c), dtype=torch.float32, device=q.device)
    check(lib().sparsek_chunk_bwd(state.cfg, c, _ptr(q), _ptr(o), _ptr(dO), _ptr(state.ws), state.ws.numel(),
                                  _ptr(dq), _ptr(dk), _ptr(dv), _ptr(du), _ptr(state.bwd_ws), state.bwd_ws.numel(),
                                  _stream()))
    return dq, dk, dv, du


def sparsek_chunk_to_decode(state, n_consumed, decode_state):
    """Fills a DecodeState with the state after the n_consumed tokens the chunks have covered."""
    check(lib().sparsek_chunk_to_decode(state.cfg, _ptr(state.buf), state.buf.numel(), int(n_consumed),
                                        _ptr(state.ws), state.ws.numel(), decode_state.cfg,
                                        _ptr(decode_state.buf), decode_state.buf.numel(), _stream()))


def sparsek_chunk_status(state):
    """(retained entries, flag word) per score row, as two int32 numpy arrays; synchronises."""
    import numpy as np

    rows = state.cfg.B * state.cfg.Gu
    counts = np.zeros(rows, np.int32)
    flags = np.zeros(rows, np.int32)
    check(lib().sparsek_chunk_status(state.cfg, _ptr(state.buf), counts.ctypes.data_as(C.c_void_p),
                                     flags.ctypes.data_as(C.c_void_p), _stream()))
    return counts, flags


class DecodeState:
    """Caller-owned decode state: a config plus one device buffer."""

    def __init__(self, B, H, Gu, d, k, w, dtype, gate_mode=0, scale=1.0, cand_cap=0, device="cuda"):
        torch = _torch()
        self.cfg = SparsekDecodeCfg(B=B, H=H, Gu=Gu, d=d, k=int(k), w=int(w), cand_cap=int(cand_cap),
                                    dtype=BF16 if dtype == torch.bfloat16 else F32,
                                    gate_mode=int(gate_mode), softmax_scale=float(scale))
        self.torch_dtype = dtype
        nbytes = lib().sparsek_decode_state_bytes(self.cfg)
        if nbytes == 0:
            raise ValueError("unsupported decode configuration")
        self.buf = torch.empty(int(nbytes), dtype=torch.uint8, device=device)


def sparsek_decode_init(state):
    check(lib().sparsek_decode_init(state.cfg, _ptr(state.buf), state.buf.numel(), _stream()))


def sparsek_decode_load(state, k, v, u, tau, death):
    n_ctx = k.shape[2]
    check(lib().sparsek_decode_load(state.cfg, _ptr(state.buf), state.buf.numel(), int(n_ctx),
                                    _ptr(k), _ptr(v), _ptr(u), _ptr(tau), _ptr(death), _stream()))


def sparsek_decode_step(state, q_new, k_new, v_new, u_new, out=None):
    torch, L = _torch(), lib()
    o = out if out is not None else torch.empty_like(q_new)
    rc = L.sparsek_decode_step(state.cfg, state.buf.data_ptr(), q_new.data_ptr(), k_new.data_ptr(), v_new.data_ptr(),
                               u_new.data_ptr(), o.data_ptr(), _raw_stream())
    if rc:
        check(rc)
    return o


def sparsek_decode_status(state):
    import numpy as np

    flags = np.zeros(state.cfg.B * state.cfg.Gu, np.int32)
    check(lib().sparsek_decode_status(state.cfg, _ptr(state.buf),
                                      flags.ctypes.data_as(C.c_void_p), _stream()))
    return flags


# ---- attention over blocks of 64 tokens that a cheap score selects ----

def _same(name, t, dtype, shape, device):
    """The tensor is contiguous, of that type and shape, and on that device."""
    if t.dtype is not dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on %s, got %s %s on %s%s" % (
            name, dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device, "" if t.is_contiguous() else " (strided)"))


def _on(device, f, *args):
    """f(*args, stream) for the device that the tensors are on, on its current stream."""
    if device.type != "cuda":
        raise ValueError("the tensors must be on the GPU, got %s" % device)
    here = _here[0]()
    if device.index == here:
        rc = f(*args, _here[1](here))
    else:
        with torch.cuda.device(device):
            rc = f(*args, _raw_stream())
    if rc:
        check(rc)


def _make_block_cfg(B, H, Hkv, n, d, top, dtype, scale):
    return SparsekBlockCfg(B=B, H=H, Hkv=Hkv, n=n, d=d, top=top, dtype=dtype, softmax_scale=scale)


def _block_kept(q, k, top, scale):
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q is [B,H,n,d] and k, v are [B,Hkv,n,d]")
    B, H, n, d = q.shape
    _same("q", q, torch.bfloat16, (B, H, n, d), q.device)
    _same("k", k, torch.bfloat16, (B, k.shape[1], n, d), q.device)
    return _kept("block", (B, H, k.shape[1], n, d, int(top), BF16, float(scale)), _make_block_cfg)


def _block_ws(cfg, query, ws, device):
    """The caller's workspace, or a new one of the size the query says (0: the configuration is refused by the call itself)."""
    if ws is None:
        return _attn_ws(cfg, query, None, device)
    if ws.device != device or not ws.is_contiguous():
        raise ValueError("ws must be contiguous and on %s" % device)
    return ws, ws.numel() * ws.element_size()


def sparsek_block_select(q, k, top, ws=None):
    """idx [B,Hkv,n,top] int32: for every query of q [B,H,n,d] (bf16) the `top` blocks of 64 keys of k [B,Hkv,n,d] behind its own with
    the largest cheap scores, ascending, padded with -1; the query heads of a key/value head share them."""
    torch = _torch()
    cfg = _block_kept(q, k, top, 1.0)
    idx = torch.empty(q.shape[0], k.shape[1], q.shape[2], max(int(top), 0), dtype=torch.int32, device=q.device)
    ws, nbytes = _block_ws(cfg, "sparsek_block_select_workspace_bytes", ws, q.device)
    _on(q.device, lib().sparsek_block_select, cfg[0], q.data_ptr(), k.data_ptr(), idx.data_ptr(), ws.data_ptr(), nbytes)
    return idx


def _block_rest(q, k, v, idx):
    if idx.dim() != 4:
        raise ValueError("idx is [B,Hkv,n,top]")
    _same("idx", idx, torch.int32, (q.shape[0], k.shape[1], q.shape[2], idx.shape[3]), q.device)
    _same("v", v, torch.bfloat16, k.shape, q.device)


def sparsek_block_attn_fwd(q, k, v, idx, scale, mass=False, ws=None):
    """o [B,H,n,d] and lse [B,H,n] fp32 of attention over every query's own block of 64 keys and the blocks that idx names; with
    mass=True also the weight that each block got, [B,Hkv,ceil(n/64)] fp32."""
    torch = _torch()
    cfg = _block_kept(q, k, idx.shape[-1], scale)
    _block_rest(q, k, v, idx)
    o = torch.empty_like(q)
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    m = torch.empty(k.shape[0], k.shape[1], -(-k.shape[2] // BLOCK_TOKENS), dtype=torch.float32, device=q.device) if mass else None
    ws, nbytes = _block_ws(cfg, "sparsek_block_attn_fwd_workspace_bytes", ws, q.device)
    _on(q.device, lib().sparsek_block_attn_fwd, cfg[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), idx.data_ptr(), o.data_ptr(),
        lse.data_ptr(), _ptr(m), ws.data_ptr(), nbytes)
    return (o, lse, m) if mass else (o, lse)


def sparsek_block_attn_bwd(q, k, v, idx, o, lse, dO, scale, ws=None):
    """dq [B,H,n,d], dk, dv [B,Hkv,n,d]: gradients of sum(dO*o) for the outputs o, lse of sparsek_block_attn_fwd, the selection held fixed."""
    torch = _torch()
    cfg = _block_kept(q, k, idx.shape[-1], scale)
    _block_rest(q, k, v, idx)
    _same("o", o, torch.bfloat16, q.shape, q.device)
    _same("dO", dO, torch.bfloat16, q.shape, q.device)
    _same("lse", lse, torch.float32, q.shape[:3], q.device)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws, nbytes = _block_ws(cfg, "sparsek_block_attn_bwd_workspace_bytes", ws, q.device)
    _on(q.device, lib().sparsek_block_attn_bwd, cfg[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), idx.data_ptr(), o.data_ptr(),
        lse.data_ptr(), dO.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), nbytes)
    return dq, dk, dv


# ---- a key/value cache in blocks of 64 tokens held in 8 bits, or in 4 ----

class _Cache:
    """What both caches are: tensors of the caller's that were checked once, and the addresses that the calls go by."""

    def _keep(self, tensors, H, scale, format, pages, d):
        B, Hkv, cap = tensors["table"].shape
        for name in self._names:
            setattr(self, name, tensors[name])
        self.B, self.H, self.Hkv, self.d, self.cap, self.device = B, int(H), Hkv, d, cap, tensors["table"].device
        self.cfg = SparsekCache8Cfg(B=B, H=int(H), Hkv=Hkv, d=d, cap=cap, pages=pages, format=format, dtype=BF16, softmax_scale=float(scale))
        self.q_shape, self.lens_shape, self.bytes = (B, int(H), d), (B,), {}
        if not lib().sparsek_cache8_attn_workspace_bytes(self.cfg, 0) and not lib().sparsek_cache4_attn_workspace_bytes(self.cfg, 0):
            raise ValueError("unsupported cache configuration")
        self._ref()

    def __setattr__(self, name, value):
        if name in self._names and hasattr(self, "cref"):   # (the calls go by the addresses taken in the constructor)
            raise AttributeError("the tensors of a %s stay; adopt() takes another table and masses" % type(self).__name__)
        object.__setattr__(self, name, value)

    def _ref(self):
        self.c = self._struct(*(getattr(self, n).data_ptr() for n in self._names))
        self.ref, self.cref = C.byref(self.cfg), C.byref(self.c)

    def adopt(self, table, mass):
        """From now on with this table and these masses (those that sparsek_cache8_evict or sparsek_cache4_evict gave)."""
        _same("table", table, torch.int32, (self.B, self.Hkv, self.cap), self.device)
        _same("mass", mass, torch.float32, (self.B, self.Hkv, self.cap), self.device)
        object.__setattr__(self, "table", table)
        object.__setattr__(self, "mass", mass)
        self._ref()


def _common(B, Hkv, d, cap, pages):
    """(name, type, shape) of the tensors that both caches have."""
    return (("ks", torch.float32, (pages,)), ("vs", torch.float32, (pages,)), ("km", torch.int8, (pages, d)), ("kms", torch.float32, (pages,)),
            ("kt", torch.bfloat16, (B, Hkv, BLOCK_TOKENS, d)), ("vt", torch.bfloat16, (B, Hkv, d, BLOCK_TOKENS)),
            ("table", torch.int32, (B, Hkv, cap)), ("mass", torch.float32, (B, Hkv, cap)))


def _empty_common(B, Hkv, d, cap, pages, device):
    """Those tensors of a cache without tokens: every row of the table has an equal share of the pages, in order."""
    got = {name: torch.zeros(*shape, dtype=dtype, device=device) for name, dtype, shape in _common(B, Hkv, d, cap, pages)}
    # (no page in two places: an append writes whole pages, and two of one page would mix their tokens)
    share = min(pages // (B * Hkv), cap) if B * Hkv > 0 else 0
    place, row = torch.arange(cap, device=device), torch.arange(B * Hkv, device=device).view(B, Hkv, 1)
    got["table"] = torch.where(place < share, row * share + place, -1).to(torch.int32)
    return got


class Cache8(_Cache):
    """The tensors of a cache (see include/sparsek.h), checked once.  The constructor takes the caller's own; Cache8.empty makes
    them: a pool of `pages` pages, of which every row of the table (a sequence's key/value head) has an equal share, in order."""
    _names, _struct = _CACHE8_TENSORS, SparsekCache8

    def __init__(self, k8, v8, ks, vs, km, kms, kt, vt, table, mass, H, scale):
        torch = _torch()
        if k8.dim() != 3 or table.dim() != 3:
            raise ValueError("k8 is [pages,64,d] and table is [B,Hkv,cap]")
        pages, T, d = k8.shape
        B, Hkv, cap = table.shape
        formats = {torch.int8: I8, torch.float8_e4m3fn: E4M3}
        if k8.dtype not in formats:
            raise ValueError("k8 must be int8 or float8_e4m3fn, got %s" % k8.dtype)
        dev = k8.device
        tensors = dict(k8=k8, v8=v8, ks=ks, vs=vs, km=km, kms=kms, kt=kt, vt=vt, table=table, mass=mass)
        for name, dtype, shape in (("k8", k8.dtype, (pages, BLOCK_TOKENS, d)), ("v8", k8.dtype, (pages, d, BLOCK_TOKENS))) + _common(B, Hkv, d, cap, pages):
            _same(name, tensors[name], dtype, shape, dev)
        self._keep(tensors, H, scale, formats[k8.dtype], pages, d)

    @classmethod
    def empty(cls, B, H, Hkv, d, cap, format=None, scale=None, pages=None, device="cuda"):
        """A cache without tokens; format torch.int8 (default) or torch.float8_e4m3fn, scale d ** -0.5 by default.  `pages` (default:
        one for every place of the table) may be fewer: places beyond a row's pages // (B * Hkv) hold -1, and blocks that become whole
        there are dropped, until the caller writes pages of their own into the table (those beyond the shares are in nobody's)."""
        torch = _torch()
        format = torch.int8 if format is None else format
        pages = B * Hkv * cap if pages is None else int(pages)
        codes = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=device).view(format)   # noqa: E731
        return cls(codes(pages, BLOCK_TOKENS, d), codes(pages, d, BLOCK_TOKENS), **_empty_common(B, Hkv, d, cap, pages, device), H=H,
                   scale=d ** -0.5 if scale is None else scale)


class Cache4(_Cache):
    """The tensors of a cache in 4 bits (see include/sparsek.h), checked once.  The constructor takes the caller's own; Cache4.empty makes
    them, as Cache8.empty does."""
    _names, _struct = _CACHE4_TENSORS, SparsekCache4

    def __init__(self, k4, v4, ke, ve, ks, vs, km, kms, kt, vt, table, mass, H, scale):
        torch = _torch()
        if km.dim() != 2 or table.dim() != 3:
            raise ValueError("km is [pages,d] and table is [B,Hkv,cap]")
        pages, d = km.shape
        B, Hkv, cap = table.shape
        tensors = dict(k4=k4, v4=v4, ke=ke, ve=ve, ks=ks, vs=vs, km=km, kms=kms, kt=kt, vt=vt, table=table, mass=mass)
        u8 = torch.uint8
        for name, dtype, shape in (("k4", u8, (pages, 32 * d)), ("v4", u8, (pages, 32 * d)), ("ke", u8, (pages, 2 * d)),
                                   ("ve", u8, (pages, 2 * d))) + _common(B, Hkv, d, cap, pages):
            _same(name, tensors[name], dtype, shape, k4.device)
        self._keep(tensors, H, scale, E2M1, pages, d)

    @classmethod
    def empty(cls, B, H, Hkv, d, cap, scale=None, pages=None, device="cuda"):
        """A cache without tokens; scale d ** -0.5 by default, pages as for Cache8.empty."""
        torch = _torch()
        pages = B * Hkv * cap if pages is None else int(pages)
        z = lambda size: torch.zeros(pages, size, dtype=torch.uint8, device=device)   # noqa: E731
        return cls(z(32 * d), z(32 * d), z(2 * d), z(2 * d), **_empty_common(B, Hkv, d, cap, pages, device), H=H, scale=d ** -0.5 if scale is None else scale)


def _cache_append(f, cache, lens, k, v, counts):
    shape = (cache.B, cache.Hkv, k.shape[2] if k.dim() == 4 else 0, cache.d)
    _same("k", k, torch.bfloat16, shape, cache.device)
    _same("v", v, torch.bfloat16, shape, cache.device)
    _same("lens", lens, torch.int32, cache.lens_shape, cache.device)
    if counts is not None:
        _same("counts", counts, torch.int32, cache.lens_shape, cache.device)
    _on(cache.device, f, cache.ref, cache.cref, lens.data_ptr(), _ptr(counts), shape[2], k.data_ptr(), v.data_ptr())


def _cache_select(f, cache, lens, q, top):
    _same("q", q, torch.bfloat16, cache.q_shape, cache.device)
    _same("lens", lens, torch.int32, cache.lens_shape, cache.device)
    idx = torch.empty(cache.B, cache.Hkv, max(int(top), 0), dtype=torch.int32, device=cache.device)
    _on(cache.device, f, cache.ref, cache.cref, lens.data_ptr(), q.data_ptr(), int(top), idx.data_ptr())
    return idx


def _cache_attn(f, need, cache, lens, q, idx, accumulate, ws):
    top = 0
    _same("q", q, torch.bfloat16, cache.q_shape, cache.device)
    _same("lens", lens, torch.int32, cache.lens_shape, cache.device)
    if idx is not None:
        top = idx.shape[-1]
        _same("idx", idx, torch.int32, (cache.B, cache.Hkv, top), cache.device)
        if top == 0:   # (a tensor without elements has no address, which would stand for all tokens: one place that names no block)
            idx, top = torch.full((cache.B, cache.Hkv, 1), -1, dtype=torch.int32, device=cache.device), 1
    o = torch.empty_like(q)
    lse = torch.empty(cache.B, cache.H, dtype=torch.float32, device=cache.device)
    if ws is None:
        nbytes = cache.bytes.get(top)
        if nbytes is None:
            nbytes = cache.bytes[top] = max(need(cache.ref, top), 256)
        if nbytes > 256 or type(cache) is Cache8:   # (in 4 bits that is no workspace at all)
            ws = torch.empty(nbytes, dtype=torch.uint8, device=cache.device)
    else:
        if ws.device != cache.device or not ws.is_contiguous():
            raise ValueError("ws must be contiguous and on %s" % cache.device)
        nbytes = ws.numel() * ws.element_size()
    _on(cache.device, f, cache.ref, cache.cref, lens.data_ptr(), q.data_ptr(), _ptr(idx), top, 1 if accumulate else 0,
        o.data_ptr(), lse.data_ptr(), _ptr(ws), nbytes)
    return o, lse


def _cache_evict(f, cache, lens, budget, sink, recent, out):
    _same("lens", lens, torch.int32, cache.lens_shape, cache.device)
    if out is None:
        out = dict(table=torch.empty_like(cache.table), mass=torch.empty_like(cache.mass), lens=torch.empty_like(lens))
    table, mass, after = out["table"], out["mass"], out["lens"]
    _same("out table", table, torch.int32, cache.table.shape, cache.device)
    _same("out mass", mass, torch.float32, cache.mass.shape, cache.device)
    _same("out lens", after, torch.int32, cache.lens_shape, cache.device)
    _on(cache.device, f, cache.ref, cache.cref, lens.data_ptr(), int(budget), int(sink), int(recent),
        table.data_ptr(), mass.data_ptr(), after.data_ptr())
    return out


def sparsek_cache8_append(cache, lens, k, v, counts=None):
    """The first counts[b] (None: all) of the new tokens k, v [B,Hkv,c,d] join the lens[b] (int32 [B]) that sequence b has; lens itself is
    the caller's to move on."""
    _cache_append(lib().sparsek_cache8_append, cache, lens, k, v, counts)


def sparsek_cache8_select(cache, lens, q, top):
    """idx [B,Hkv,top] int32: the places in the table of the `top` whole blocks behind the own block of the query q [B,H,d] at position
    lens - 1 with the largest cheap scores, ascending, padded with -1."""
    return _cache_select(lib().sparsek_cache8_select, cache, lens, q, top)


def sparsek_cache8_attn(cache, lens, q, idx=None, accumulate=False, ws=None):
    """o [B,H,d] and lse [B,H] fp32 of the query q [B,H,d] at position lens - 1 over all tokens (idx None), or over its own block and
    those of idx [B,Hkv,top] (top 0: its own block only); accumulate=True adds the weights to cache.mass."""
    return _cache_attn(lib().sparsek_cache8_attn, lib().sparsek_cache8_attn_workspace_bytes, cache, lens, q, idx, accumulate, ws)


def sparsek_cache8_evict(cache, lens, budget, sink=1, recent=1, out=None):
    """Sequences with more than `budget` whole blocks keep the first `sink`, the last `recent` and the heaviest of the others.  Returns
    dict(table, mass, lens), new tensors or those of `out`; cache.adopt(table, mass) makes the cache go on with them."""
    return _cache_evict(lib().sparsek_cache8_evict, cache, lens, budget, sink, recent, out)


def sparsek_cache4_append(cache, lens, k, v, counts=None):
    """As sparsek_cache8_append, into a Cache4."""
    _cache_append(lib().sparsek_cache4_append, cache, lens, k, v, counts)


def sparsek_cache4_select(cache, lens, q, top):
    """As sparsek_cache8_select, from a Cache4."""
    return _cache_select(lib().sparsek_cache4_select, cache, lens, q, top)


def sparsek_cache4_attn(cache, lens, q, idx=None, accumulate=False, ws=None):
    """As sparsek_cache8_attn, over a Cache4."""
    return _cache_attn(lib().sparsek_cache4_attn, lib().sparsek_cache4_attn_workspace_bytes, cache, lens, q, idx, accumulate, ws)


def sparsek_cache4_evict(cache, lens, budget, sink=1, recent=1, out=None):
    """As sparsek_cache8_evict, from a Cache4."""
    return _cache_evict(lib().sparsek_cache4_evict, cache, lens, budget, sink, recent, out)


def sparsek_cache4_read(cache, lens, begin, n, out=None):
    """k, v [B,Hkv,n,d] bf16: tokens begin .. begin + n - 1 of every sequence as they are attended, zeros behind its end; new tensors or those
    of `out`."""
    _same("lens", lens, torch.int32, cache.lens_shape, cache.device)
    shape = (cache.B, cache.Hkv, int(n), cache.d)
    if out is None:
        out = cache.kt.new_empty((2, cache.B, cache.Hkv, max(int(n), 0), cache.d)).unbind()
    else:
        for name, t in zip(("out k", "out v"), out):
            _same(name, t, torch.bfloat16, shape, cache.device)
    k, v = out
    _on(cache.device, lib().sparsek_cache4_read, cache.ref, cache.cref, lens.data_ptr(), int(begin), int(n), k.data_ptr(), v.data_ptr())
    return k, v


# ---- norms of queries and keys with rotary positions ----

def _make_rope_cfg(B, H, Hkv, n, d, rot, axes, interleaved, norm, dtype, eps, q, k, dq, dk):
    return SparsekRopeCfg(B=B, H=H, Hkv=Hkv, n=n, d=d, rot=rot, axes=axes, interleaved=interleaved, norm=norm, dtype=dtype, eps=eps,
                          **{name: SparsekRopeStrides(*s) for name, s in (("q", q), ("k", k), ("dq", dq), ("dk", dk))})


def _heads_of(name, t, dtype, shape, device):
    """The strides of batch, token and head of a tensor [B,n,heads,d] whose channels are contiguous (those of one place count as 0)."""
    if t.dtype is not dtype or t.shape != shape or t.device != device:
        raise ValueError("%s must be a %s tensor of shape %s on %s, got %s %s on %s" % (
            name, dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device))
    if t.stride(3) != 1:
        raise ValueError("the channels of %s must be contiguous" % name)
    return tuple(t.stride(x) if t.shape[x] > 1 else 0 for x in range(3))


def _seen(t):
    """What the checks of a tensor go by."""
    return (t.dtype, t.shape, t.stride(), t.device) if t is not None else None


_ropes = {}   # configurations by what their tensors look like: a call on tensors like an earlier one's needs no more checks


def _rope_kept(q, k, pos, freq, axis, interleaved, norm, qw, kw, eps, grads=(None, None)):
    key = (_seen(q), _seen(k), _seen(pos), _seen(freq), _seen(axis), _seen(qw), _seen(kw), _seen(grads[0]), _seen(grads[1]), interleaved, norm, eps)
    got = _ropes.get(key)
    if got is None:
        got = _rope_checked(q, k, pos, freq, axis, interleaved, norm, qw, kw, eps, grads)
        if len(_ropes) >= _CFG_KEPT:
            _ropes.clear()
        _ropes[key] = got
    return got


def _rope_checked(q, k, pos, freq, axis, interleaved, norm, qw, kw, eps, grads):
    torch = _torch()
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError("q is [B,n,H,d] and k is [B,n,Hkv,d]")
    B, n, H, d = q.shape
    Hkv, dev = k.shape[2] if k is not None else 0, q.device
    dtype = _dtype_code(q)
    none = (0, 0, 0)
    strides = [_heads_of(name, t, q.dtype, (B, n, heads, d), dev) if t is not None else none
               for name, t, heads in (("q", q, H), ("k", k, Hkv), ("dq", grads[0], H), ("dk", grads[1], Hkv))]
    rot, axes = 2 * freq.shape[0] if freq is not None else 0, 1
    if rot:
        if pos is None or pos.dim() != 3:
            raise ValueError("pos is [axes,B,n]")
        axes = pos.shape[0]
        _same("pos", pos, torch.int32, (axes, B, n), dev)
        _same("freq", freq, torch.float32, (rot // 2,), dev)
        if axis is not None:
            _same("axis", axis, torch.int32, (rot // 2,), dev)
    for name, w in (("qw", qw), ("kw", kw)):
        if w is not None:
            if not norm:
                raise ValueError("%s without norm" % name)
            _same(name, w, torch.float32, (d,), dev)
    return _kept("rope", (B, H, Hkv, n, d, rot, axes, int(bool(interleaved)), int(bool(norm)), dtype, float(eps), *strides), _make_rope_cfg)


def sparsek_rope_fwd(q, k, pos, freq, axis=None, interleaved=False, norm=False, qw=None, kw=None, eps=1e-6, out=None):
    """Queries q [B,n,H,d] and keys k [B,n,Hkv,d] (any strides of batch, token and head; k None: queries alone) with each head's norm, if
    norm, weighted by qw, kw [d] fp32, if given, and turned by their positions: pair p by pos[axis[p]] * freq[p] (pos [axes,B,n] int32, freq
    [rot/2] fp32 or None, axis [rot/2] int32, None: the first).  Returns qo [B,H,n,d] and ko [B,Hkv,n,d] (None without k), new or those of `out`."""
    cfg = _rope_kept(q, k, pos, freq, axis, interleaved, norm, qw, kw, eps)
    B, n, H, d = q.shape
    if out is None:
        qo, ko = q.new_empty((B, H, n, d)), k.new_empty((B, k.shape[2], n, d)) if k is not None else None
    else:
        qo, ko = out
        _same("out q", qo, q.dtype, (B, H, n, d), q.device)
        if k is not None:
            _same("out k", ko, q.dtype, (B, k.shape[2], n, d), q.device)
    _on(q.device, lib().sparsek_rope_fwd, cfg[0], q.data_ptr(), _ptr(k), _ptr(pos), _ptr(freq), _ptr(axis), _ptr(qw), _ptr(kw), qo.data_ptr(),
        _ptr(ko) if k is not None else None)
    return qo, ko


def sparsek_rope_bwd(q, k, pos, freq, dqo, dko, axis=None, interleaved=False, norm=False, qw=None, kw=None, eps=1e-6, out=None, ws=None):
    """dq [B,n,H,d], dk [B,n,Hkv,d], dqw, dkw [d] fp32 (None where there is no such weight): gradients of sum(dqo*qo) + sum(dko*ko) for the
    outputs of sparsek_rope_fwd on the same arguments.  out: (dq, dk) to write to, in any strides (slices of a fused gradient)."""
    B, n, H, d = q.shape
    if out is None:
        out = q.new_empty(q.shape), k.new_empty(k.shape) if k is not None else None
    dq, dk = out
    if (dk is None) != (k is None) or (dko is None) != (k is None):
        raise ValueError("k, dko and dk go together")
    cfg = _rope_kept(q, k, pos, freq, axis, interleaved, norm, qw, kw, eps, out)
    _same("dqo", dqo, q.dtype, (B, H, n, d), q.device)
    if k is not None:
        _same("dko", dko, q.dtype, (B, k.shape[2], n, d), q.device)
    dqw = torch.empty_like(qw) if qw is not None else None
    dkw = torch.empty_like(kw) if kw is not None and k is not None else None
    nbytes = 0
    if dqw is not None or dkw is not None:
        ws, nbytes = _block_ws(cfg, "sparsek_rope_bwd_workspace_bytes", ws, q.device)
    else:
        ws = None
    _on(q.device, lib().sparsek_rope_bwd, cfg[0], q.data_ptr(), _ptr(k), _ptr(pos), _ptr(freq), _ptr(axis), _ptr(qw), _ptr(kw), dqo.data_ptr(),
        _ptr(dko), dq.data_ptr(), _ptr(dk), _ptr(dqw), _ptr(dkw), _ptr(ws), nbytes)
    return dq, dk, dqw, dkw
