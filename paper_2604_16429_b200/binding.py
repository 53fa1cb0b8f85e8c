"""Thin ctypes binding of the C ABI in ``include/mosaic_bsa.h``.

Argument marshalling only: every step of the path runs in the CUDA library.  torch is
used for device memory and streams.  There is no CPU fallback: if the library is missing
or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import math
import os
import struct
import threading
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmosaic_bsa.so")
_lib = None

OP_SELECT, OP_FWD, OP_BWD, OP_FWD_BRANCHES, OP_BWD_BRANCHES = 0, 1, 2, 3, 4
EXPORTS = ("mosaic_bsa_workspace_bytes", "mosaic_bsa_select", "mosaic_bsa_fwd", "mosaic_bsa_bwd",
           "mosaic_bsa_last_status", "mosaic_bsa_strerror", "mosaic_bsa_select_static",
           "mosaic_bsa_descriptor_encodes", "mosaic_bsa_fwd_branches", "mosaic_bsa_bwd_branches", "mosaic_bsa_rope",
           "mosaic_bsa_rotary_freqs", "mosaic_bsa_rotary", "mosaic_bsa_qk_norm", "mosaic_bsa_qk_norm_workspace_bytes",
           "mosaic_bsa_qk_norm_bwd", "mosaic_bsa_window_workspace_bytes", "mosaic_bsa_window_fwd",
           "mosaic_bsa_window_bwd", "mosaic_bsa_window_decode")
STATIC_SCRATCH_BYTES = 4 << 20
FLAG_LOCAL_GROUPS = 1
FLAG_FP16 = 2
FLAG_FP32, FLAG_HALF_PAIRS, FLAG_INVERSE, FLAG_ROLLING = 4, 8, 16, 32
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS, ROTARY_BANDS = 0, 1, 2, 3, 4


class MosaicError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


class _Params(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("nlat", ctypes.c_int32), ("nlon", ctypes.c_int32),
                ("d", ctypes.c_int32), ("bh", ctypes.c_int32), ("bw", ctypes.c_int32),
                ("rlat", ctypes.c_int32), ("rlon", ctypes.c_int32), ("topk", ctypes.c_int32),
                ("scale", ctypes.c_float), ("flags", ctypes.c_uint32), ("Hkv", ctypes.c_int32)]


class _View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("sb", ctypes.c_int64), ("sh", ctypes.c_int64), ("sn", ctypes.c_int64)]


class _RotaryParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("N", ctypes.c_int32),
                ("d", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("amplitude", ctypes.c_float), ("eps", ctypes.c_float)]


class _RotaryScaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("theta", ctypes.c_double),
                ("factor", ctypes.c_double), ("length", ctypes.c_double), ("fast", ctypes.c_double),
                ("slow", ctypes.c_double)]


class _WindowParams(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("Nq", ctypes.c_int32),
                ("Nk", ctypes.c_int32), ("d", ctypes.c_int32), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


@dataclass(frozen=True)
class Params:
    B: int
    H: int
    nlat: int
    nlon: int
    d: int = 64
    bh: int = 8
    bw: int = 8
    rlat: int = 1
    rlon: int = 1
    topk: int = 8
    scale: float = 0.0
    flags: int = 0
    Hkv: int = 0          # heads of K and V (grouped-query attention); 0 = H

    @property
    def kv_heads(self): return self.Hkv or self.H
    @property
    def N(self): return self.nlat * self.nlon
    @property
    def m(self): return (self.nlat // self.bh) * (self.nlon // self.bw)
    @property
    def U(self): return self.B * self.H

    def c(self):
        return _Params(self.B, self.H, self.nlat, self.nlon, self.d, self.bh, self.bw, self.rlat, self.rlon,
                       self.topk, self.scale, self.flags, self.Hkv)

    @staticmethod
    def from_workload(w, **over):
        kw = dict(B=w.B, H=w.H, nlat=w.nlat, nlon=w.nlon, d=w.d, bh=w.bh, bw=w.bw, rlat=w.rlat, rlon=w.rlon,
                  topk=w.topk, flags=(FLAG_LOCAL_GROUPS if getattr(w, "local_groups", False) else 0)
                  | (FLAG_FP16 if getattr(w, "f16", False) else 0),
                  Hkv=getattr(w, "Hkv", 0))
        kw.update(over)
        return Params(**kw)


def lib():
    """Load the CUDA library; fails loudly if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_16429_b200.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p, fp = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
        pp = ctypes.POINTER(_Params)
        L.mosaic_bsa_workspace_bytes.restype = ctypes.c_size_t
        L.mosaic_bsa_workspace_bytes.argtypes = [pp, ctypes.c_int]
        L.mosaic_bsa_select.restype = ctypes.c_int
        L.mosaic_bsa_select.argtypes = [pp, vp, vp, i32p, vp, ctypes.c_size_t, vp]
        L.mosaic_bsa_select_static.restype = ctypes.c_int
        L.mosaic_bsa_select_static.argtypes = [pp, vp, vp, i32p, vp]
        L.mosaic_bsa_fwd.restype = ctypes.c_int
        L.mosaic_bsa_fwd.argtypes = [pp, vp, vp, vp, i32p, vp, fp, vp, ctypes.c_size_t, vp]
        L.mosaic_bsa_fwd_branches.restype = ctypes.c_int
        L.mosaic_bsa_fwd_branches.argtypes = [pp, vp, vp, vp, i32p, fp, vp, fp, fp, vp, ctypes.c_size_t, vp]
        L.mosaic_bsa_bwd_branches.restype = ctypes.c_int
        L.mosaic_bsa_bwd_branches.argtypes = [pp, vp, vp, vp, i32p, fp, vp, vp, vp, vp, fp, vp, ctypes.c_size_t, vp]
        L.mosaic_bsa_rope.restype = ctypes.c_int
        L.mosaic_bsa_rope.argtypes = [pp, vp, vp, fp, ctypes.c_float, vp, vp, vp]
        L.mosaic_bsa_bwd.restype = ctypes.c_int
        L.mosaic_bsa_bwd.argtypes = [pp, vp, vp, vp, vp, fp, vp, i32p, vp, vp, vp, vp, ctypes.c_size_t, vp]
        vw = rp = vp  # pointers to a view, to a parameter block
        L.mosaic_bsa_rotary_freqs.restype = ctypes.c_int
        L.mosaic_bsa_rotary_freqs.argtypes = [ctypes.POINTER(_RotaryScaling), vp]
        L.mosaic_bsa_rotary.restype = ctypes.c_int
        L.mosaic_bsa_rotary.argtypes = [rp, vw, vw, vp, ctypes.c_int64, vp, vw, vw, vp]
        L.mosaic_bsa_qk_norm.restype = ctypes.c_int
        L.mosaic_bsa_qk_norm.argtypes = [rp, vw, vw, fp, fp, vp, ctypes.c_int64, vp, vw, vw, vp]
        L.mosaic_bsa_qk_norm_workspace_bytes.restype = ctypes.c_size_t
        L.mosaic_bsa_qk_norm_workspace_bytes.argtypes = [rp]
        L.mosaic_bsa_qk_norm_bwd.restype = ctypes.c_int
        L.mosaic_bsa_qk_norm_bwd.argtypes = [rp, vw, vw, fp, fp, vp, ctypes.c_int64, vp, vw, vw, vw, vw, fp, fp, vp,
                                             ctypes.c_size_t, vp]
        wp = vp
        L.mosaic_bsa_window_workspace_bytes.restype = ctypes.c_size_t
        L.mosaic_bsa_window_workspace_bytes.argtypes = [wp, ctypes.c_int]
        L.mosaic_bsa_window_fwd.restype = ctypes.c_int
        L.mosaic_bsa_window_fwd.argtypes = [wp, vw, vw, vw, i32p, i32p, vw, fp, vp, ctypes.c_size_t, vp]
        L.mosaic_bsa_window_bwd.restype = ctypes.c_int
        L.mosaic_bsa_window_bwd.argtypes = [wp, vw, vw, vw, vw, fp, vw, i32p, i32p, vw, vw, vw, vp, ctypes.c_size_t, vp]
        L.mosaic_bsa_window_decode.restype = ctypes.c_int
        L.mosaic_bsa_window_decode.argtypes = [wp, vw, vw, vw, i32p, vw, fp, vp]
        L.mosaic_bsa_last_status.restype = ctypes.c_int
        L.mosaic_bsa_last_status.argtypes = [vp, vp]
        L.mosaic_bsa_descriptor_encodes.restype = ctypes.c_longlong
        L.mosaic_bsa_descriptor_encodes.argtypes = []
        L.mosaic_bsa_strerror.restype = ctypes.c_char_p
        L.mosaic_bsa_strerror.argtypes = [ctypes.c_int]
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().mosaic_bsa_strerror(int(code)).decode()


def workspace_bytes(p: Params, op: int) -> int:
    pc = p.c()
    return int(lib().mosaic_bsa_workspace_bytes(ctypes.byref(pc), op))


def _stream(stream) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return int(s.cuda_stream)


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _chk_qkv(p: Params, *ts, heads=None):
    h = p.H if heads is None else heads
    dt = torch.float16 if p.flags & FLAG_FP16 else torch.bfloat16
    for t in ts:
        if t.dtype != dt or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != (p.B, h, p.N, p.d):
            raise ValueError(f"expected contiguous cuda {dt} [{p.B},{h},{p.N},{p.d}], got {t.dtype} {tuple(t.shape)}")


def alloc_workspace(p: Params, op: int, device="cuda") -> torch.Tensor:
    n = workspace_bytes(p, op)
    if n == 0:
        raise MosaicError(-1, "mosaic_bsa_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _on(stream, make, *args, **kw):
    """make(*args, **kw), a tensor that only the call itself uses, from the memory of the stream that the call runs on.  (The current
    stream's may still be read or written by what is queued there, and nothing orders `stream` behind that.)"""
    if stream is None:
        return make(*args, **kw)
    with torch.cuda.stream(stream):
        return make(*args, **kw)


def _new(stream, make, *args, **kw):
    """The same for a tensor that the call returns: once freed, not handed out again before the caller's stream has passed that."""
    if stream is None:
        return make(*args, **kw)
    t = _on(stream, make, *args, **kw)
    t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _like(t, stream):
    return torch.empty_like(t) if stream is None else _new(stream, torch.empty_like, t)


def mosaic_bsa_select(p: Params, q, k, block_idx=None, ws=None, stream=None):
    _chk_qkv(p, q)
    _chk_qkv(p, k, heads=p.kv_heads)
    if block_idx is None:
        block_idx = _new(stream, torch.empty, (p.B, p.H, p.m, p.topk), dtype=torch.int32, device=q.device)
    if ws is None:
        ws = _on(stream, alloc_workspace, p, OP_SELECT, q.device)
    pc = p.c()
    rc = lib().mosaic_bsa_select(ctypes.byref(pc), _ptr(q), _ptr(k), _ptr(block_idx), _ptr(ws), ws.numel(),
                                 _stream(stream))
    if rc:
        raise MosaicError(rc, "mosaic_bsa_select")
    return block_idx


def mosaic_bsa_select_static(p: Params, q, k, block_idx=None, stream=None):
    """Selection through the entry point that allocates nothing (scratch inside the library image).
    Only `block_idx` is created here when the caller passes none."""
    _chk_qkv(p, q)
    _chk_qkv(p, k, heads=p.kv_heads)
    if block_idx is None:
        block_idx = _new(stream, torch.empty, (p.B, p.H, p.m, p.topk), dtype=torch.int32, device=q.device)
    pc = p.c()
    rc = lib().mosaic_bsa_select_static(ctypes.byref(pc), _ptr(q), _ptr(k), _ptr(block_idx), _stream(stream))
    if rc:
        raise MosaicError(rc, "mosaic_bsa_select_static")
    return block_idx


def mosaic_bsa_fwd(p: Params, q, k, v, block_idx, o=None, lse=None, ws=None, stream=None):
    _chk_qkv(p, q)
    _chk_qkv(p, k, v, heads=p.kv_heads)
    if o is None:
        o = _like(q, stream)
    if lse is None:
        lse = _new(stream, torch.empty, (p.B, p.H, p.N), dtype=torch.float32, device=q.device)
    if ws is None:
        ws = _on(stream, alloc_workspace, p, OP_FWD, q.device)
    pc = p.c()
    rc = lib().mosaic_bsa_fwd(ctypes.byref(pc), _ptr(q), _ptr(k), _ptr(v), _ptr(block_idx), _ptr(o), _ptr(lse),
                              _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise MosaicError(rc, "mosaic_bsa_fwd")
    return o, lse


def mosaic_bsa_fwd_branches(p: Params, q, k, v, block_idx, gates, o=None, lse_fg=None, lse_l=None, ws=None, stream=None):
    """Three-branch form: gated sum of the compression, selection and local branches.  `gates` is
    [B, H, N, 3] fp32 (compression, selection, local).  Returns (o, lse_fg, lse_l)."""
    _chk_qkv(p, q)
    _chk_qkv(p, k, v, heads=p.kv_heads)
    if gates.dtype != torch.float32 or not gates.is_contiguous() or tuple(gates.shape) != (p.B, p.H, p.N, 3):
        raise ValueError(f"expected contiguous cuda fp32 gates [{p.B},{p.H},{p.N},3]")
    o = _like(q, stream) if o is None else o
    lse_fg = _new(stream, torch.empty, (p.B, p.H, p.N), dtype=torch.float32, device=q.device) if lse_fg is None else lse_fg
    lse_l = _new(stream, torch.empty, (p.B, p.H, p.N), dtype=torch.float32, device=q.device) if lse_l is None else lse_l
    if ws is None:
        ws = _on(stream, alloc_workspace, p, OP_FWD_BRANCHES, q.device)
    pc = p.c()
    rc = lib().mosaic_bsa_fwd_branches(ctypes.byref(pc), _ptr(q), _ptr(k), _ptr(v), _ptr(block_idx), _ptr(gates), _ptr(o),
                                       _ptr(lse_fg), _ptr(lse_l), _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise MosaicError(rc, "mosaic_bsa_fwd_branches")
    return o, lse_fg, lse_l


def mosaic_bsa_bwd(p: Params, q, k, v, o, lse, d_o, block_idx, dq=None, dk=None, dv=None, ws=None, stream=None):
    _chk_qkv(p, q, o, d_o)
    _chk_qkv(p, k, v, heads=p.kv_heads)
    dq = _like(q, stream) if dq is None else dq
    dk = _like(k, stream) if dk is None else dk
    dv = _like(k, stream) if dv is None else dv
    if ws is None:
        ws = _on(stream, alloc_workspace, p, OP_BWD, q.device)
    pc = p.c()
    rc = lib().mosaic_bsa_bwd(ctypes.byref(pc), _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(lse), _ptr(d_o),
                              _ptr(block_idx), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise MosaicError(rc, "mosaic_bsa_bwd")
    return dq, dk, dv


def mosaic_bsa_bwd_branches(p: Params, q, k, v, block_idx, gates, d_o, dq=None, dk=None, dv=None, dgates=None, ws=None,
                            stream=None):
    """Backward of the three-branch form.  Returns (dq, dk, dv, dgates); dgates is [B, H, N, 3] fp32."""
    _chk_qkv(p, q, d_o)
    _chk_qkv(p, k, v, heads=p.kv_heads)
    if gates.dtype != torch.float32 or not gates.is_contiguous() or tuple(gates.shape) != (p.B, p.H, p.N, 3):
        raise ValueError(f"expected contiguous cuda fp32 gates [{p.B},{p.H},{p.N},3]")
    dq = _like(q, stream) if dq is None else dq
    dk = _like(k, stream) if dk is None else dk
    dv = _like(k, stream) if dv is None else dv
    dgates = _like(gates, stream) if dgates is None else dgates
    if ws is None:
        ws = _on(stream, alloc_workspace, p, OP_BWD_BRANCHES, q.device)
    pc = p.c()
    rc = lib().mosaic_bsa_bwd_branches(ctypes.byref(pc), _ptr(q), _ptr(k), _ptr(v), _ptr(block_idx), _ptr(gates), _ptr(d_o),
                                       _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dgates), _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise MosaicError(rc, "mosaic_bsa_bwd_branches")
    return dq, dk, dv, dgates


def mosaic_bsa_rope(p: Params, q, k, pos, theta=10000.0, q_out=None, k_out=None, stream=None):
    """2-D rotary position embedding of q and k; pos is [N, 2] fp32 (longitude, latitude in radians).
    Returns (q_out, k_out)."""
    _chk_qkv(p, q)
    _chk_qkv(p, k, heads=p.kv_heads)
    if pos.dtype != torch.float32 or not pos.is_cuda or not pos.is_contiguous() or tuple(pos.shape) != (p.N, 2):
        raise ValueError(f"expected contiguous cuda fp32 positions [{p.N},2]")
    q_out = _like(q, stream) if q_out is None else q_out
    k_out = _like(k, stream) if k_out is None else k_out
    pc = p.c()
    rc = lib().mosaic_bsa_rope(ctypes.byref(pc), _ptr(q), _ptr(k), _ptr(pos), float(theta), _ptr(q_out), _ptr(k_out),
                               _stream(stream))
    if rc:
        raise MosaicError(rc, "mosaic_bsa_rope")
    return q_out, k_out


def mosaic_bsa_last_status(ws, stream=None) -> int:
    return int(lib().mosaic_bsa_last_status(_ptr(ws), _stream(stream)))


def descriptor_encodes() -> int:
    return int(lib().mosaic_bsa_descriptor_encodes())


def check_status(ws, where: str, stream=None):
    st = mosaic_bsa_last_status(ws, stream)
    if st:
        raise MosaicError(st, where + " (device status)")


def from_bits(bits, device="cuda", f16=False) -> torch.Tensor:
    """uint16 bit patterns (numpy) -> bf16 (or, with f16, float16) tensor on `device`, bit for bit."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.float16 if f16 else torch.bfloat16)


def default_scale(d: int) -> float:
    return 1.0 / math.sqrt(d)


# ---- operators on token sequences: strided tensors [B, heads, tokens, d] ---------------------------------------------
_STORAGE = {torch.bfloat16: 0, torch.float16: FLAG_FP16, torch.float32: FLAG_FP32}


@dataclass(frozen=True)
class RotaryParams:
    """What a model fixes of its rotary positions (the sizes come from the tensors)."""
    d: int
    rot_dim: int = -1          # channels that turn, -1: all of them
    half: bool = False         # pairs (i, i + rot_dim/2) instead of (2i, 2i+1)
    amplitude: float = 1.0     # factor of the turned channels
    theta: float = 10000.0     # the rest is what `rotary_freqs` reads
    scaling: int = ROTARY_PLAIN
    factor: float = 1.0
    length: float = 0.0        # positions the model was trained on (ROTARY_PARTS, ROTARY_BANDS)
    fast: float = 32.0
    slow: float = 1.0

    @property
    def rot(self): return self.d if self.rot_dim < 0 else self.rot_dim


def rotary_freqs(rp: RotaryParams, device="cuda") -> torch.Tensor:
    """Radians per position of the turned pairs, [rot_dim/2] fp64 on `device`: made once, passed to every call."""
    out = torch.empty(max(rp.rot // 2, 1), dtype=torch.float64)
    sc = _RotaryScaling(rp.scaling, rp.rot, rp.theta, rp.factor, rp.length, rp.fast, rp.slow)
    rc = lib().mosaic_bsa_rotary_freqs(ctypes.byref(sc), out.data_ptr())
    if rc:
        raise MosaicError(rc, "mosaic_bsa_rotary_freqs")
    return out.to(device)


# Small calls are as long as what happens here before the launch (a rotation of 64 tokens: 24 us with a stream object, device
# objects and a ctypes structure made per argument), hence the plain comparisons, and the parameter block and all views of a call
# written at once into a buffer that the thread keeps.
class _Block(threading.local):
    def __init__(self):
        self.buf = (ctypes.c_int64 * 48)()
        self.at = ctypes.addressof(self.buf)


_block = _Block()
# (both parameter blocks are 40 bytes long with their padding, a view is 32)
_rotary_pack = {n: struct.Struct("=6iI2f4x%dq" % (4 * n)).pack_into for n in (0, 4, 6)}
_window_pack = {n: struct.Struct("=8ifI%dq" % (4 * n)).pack_into for n in (0, 4, 8)}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


_RANGE = (struct.error, OverflowError)


def _out_of_range(e):
    return ValueError(f"a parameter is out of range: {e}")


def _params_block(layout, p):
    """Address of a parameter block alone."""
    try:
        layout(_block.buf, 0, *p)
    except _RANGE as e:
        raise _out_of_range(e) from None
    return _block.at


def _bad(name, t, what):
    return ValueError(f"{name}: expected {what}, got {t.dtype} {tuple(t.shape)} on {t.device} with strides {t.stride()}")


def _view(name, t, shape, dtype, index):
    """`t` as a strided tensor of `shape` and `dtype` on cuda device `index`, its rows contiguous."""
    st = t.stride()
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or st[3] != 1:
        raise _bad(name, t, f"{dtype} {tuple(shape)} on cuda:{index} with contiguous rows")
    return t.data_ptr(), st[0], st[1], st[2]


def _out(name, t, shape, dtype, index):
    """The same for an output, which may not write a place twice."""
    v = _view(name, t, shape, dtype, index)
    if (v[1] == 0 and shape[0] > 1) or (v[2] == 0 and shape[1] > 1) or (v[3] == 0 and shape[2] > 1):
        raise _bad(name, t, "rows that do not overlap")
    return v


def _flat(name, t, shape, dtype, index):
    """Pointer of a contiguous tensor."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or not t.is_contiguous():
        raise _bad(name, t, f"contiguous {dtype} {tuple(shape)} on cuda:{index}")
    return t.data_ptr()


def _chk_seq(q, k):
    """The device of q [B,H,N,d] and k [B,Hkv,Nk,d]."""
    index = q.get_device()
    if q.dim() != 4 or k.dim() != 4 or index < 0 or q.dtype not in _STORAGE:
        raise ValueError(f"expected cuda tensors [B, heads, tokens, d] in bf16, fp16 or fp32, got {q.dtype} {tuple(q.shape)} on "
                         f"{q.device} and {tuple(k.shape)}")
    return index


def _floats(n, index, stream):
    return torch.empty(n, dtype=torch.float32, device=index) if stream is None else _new(stream, _floats, n, index, None)


def _scratch(n, name, index, ws, stream):
    """The caller's workspace, or one of n bytes."""
    if ws is not None:
        if ws.get_device() != index or ws.dtype is not torch.uint8 or not ws.is_contiguous():
            raise _bad("ws", ws, f"contiguous uint8 on cuda:{index}")
        return ws
    if n == 0:
        raise MosaicError(-1, name)
    return torch.empty(n, dtype=torch.uint8, device=index) if stream is None else _on(stream, _scratch, n, name, index, None, None)


def _call(name, index, stream, *args):
    """The entry point on the tensors' own device, on `stream` or that device's current one."""
    if stream is None:
        raw = _raw_stream(index)
    else:
        if stream.device_index != index:
            raise ValueError(f"the stream belongs to cuda:{stream.device_index}, the tensors are on cuda:{index}")
        raw = stream.cuda_stream
    fn = getattr(_lib or lib(), name)
    if torch.cuda.current_device() == index:
        rc = fn(*args, raw)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, raw)
    if rc:
        raise MosaicError(rc, name)


def _rotary_params(rp, q, k, flags, eps):
    """(device, parameters, shape of q, shape of k)"""
    index = _chk_seq(q, k)
    B, H, N, _ = q.shape
    Hkv = k.shape[1]
    d = rp.d
    return index, (B, H, Hkv, N, d, rp.rot, _STORAGE[q.dtype] | (FLAG_HALF_PAIRS if rp.half else 0) | flags, rp.amplitude,
                   eps), (B, H, N, d), (B, Hkv, N, d)


def _positions(rp, pos, freqs, shape, index):
    """(pointer, stride) of the positions, and the frequencies' pointer."""
    rot = rp.rot
    if rot == 0:
        return 0, 0, 0
    B, _, N, _ = shape
    if pos.dtype is not torch.int64 or pos.get_device() != index or (pos.shape != (B, N) and pos.shape != (N,)) or (
            N > 1 and pos.stride(-1) != 1):
        raise _bad("pos", pos, f"int64 [{N}] or [{B},{N}] on cuda:{index}")
    return (pos.data_ptr(), pos.stride(0) if B > 1 and pos.dim() == 2 else 0,
            _flat("freqs", freqs, (rot // 2,), torch.float64, index))


def mosaic_bsa_rotary(rp: RotaryParams, q, k, pos, freqs, inverse=False, q_out=None, k_out=None, stream=None):
    """Rotary positions of q [B,H,N,d] and k [B,Hkv,N,d] by token index; pos [N] or [B,N] int64, freqs from `rotary_freqs`.
    `inverse` turns back (the transpose: what a backward applies to the gradients).  Returns (q_out, k_out)."""
    index, p, sq, sk = _rotary_params(rp, q, k, FLAG_INVERSE if inverse else 0, 0.0)
    t = q.dtype
    vq, vk = _view("q", q, sq, t, index), _view("k", k, sk, t, index)
    at, step, fr = _positions(rp, pos, freqs, sq, index)
    q_out = _like(q, stream) if q_out is None else q_out
    k_out = _like(k, stream) if k_out is None else k_out
    block = _block
    a = block.at
    try:
        _rotary_pack[4](block.buf, 0, *p, *vq, *vk, *_out("q_out", q_out, sq, t, index), *_out("k_out", k_out, sk, t, index))
    except _RANGE as e:
        raise _out_of_range(e) from None
    _call("mosaic_bsa_rotary", index, stream, a, a + 40, a + 72, at, step, fr, a + 104, a + 136)
    return q_out, k_out


def mosaic_bsa_qk_norm(rp: RotaryParams, q, k, wq, wk, pos=None, freqs=None, eps=1e-6, q_out=None, k_out=None, stream=None):
    """Root-mean-square norm of every head of q and k (weights wq, wk [d] fp32), then the rotation, in one pass; with
    rp.rot_dim 0 the norm alone.  Returns (q_out, k_out)."""
    index, p, sq, sk = _rotary_params(rp, q, k, 0, eps)
    t, f32, w = q.dtype, torch.float32, (rp.d,)
    vq, vk = _view("q", q, sq, t, index), _view("k", k, sk, t, index)
    at, step, fr = _positions(rp, pos, freqs, sq, index)
    q_out = _like(q, stream) if q_out is None else q_out
    k_out = _like(k, stream) if k_out is None else k_out
    block = _block
    a = block.at
    try:
        _rotary_pack[4](block.buf, 0, *p, *vq, *vk, *_out("q_out", q_out, sq, t, index), *_out("k_out", k_out, sk, t, index))
    except _RANGE as e:
        raise _out_of_range(e) from None
    _call("mosaic_bsa_qk_norm", index, stream, a, a + 40, a + 72, _flat("wq", wq, w, f32, index), _flat("wk", wk, w, f32, index), at,
          step, fr, a + 104, a + 136)
    return q_out, k_out


def qk_norm_workspace_bytes(rp: RotaryParams, q, k) -> int:
    return int(lib().mosaic_bsa_qk_norm_workspace_bytes(_params_block(_rotary_pack[0], _rotary_params(rp, q, k, 0, 0.0)[1])))


def mosaic_bsa_qk_norm_bwd(rp: RotaryParams, q, k, wq, wk, pos, freqs, d_q_out, d_k_out, eps=1e-6, dq=None, dk=None, dwq=None,
                           dwk=None, ws=None, stream=None):
    """Backward of mosaic_bsa_qk_norm from its inputs and its outputs' gradients.  Returns (dq, dk, dwq, dwk); the weights'
    gradients are [d] fp32."""
    index, p, sq, sk = _rotary_params(rp, q, k, 0, eps)
    t, f32, w = q.dtype, torch.float32, (rp.d,)
    vq, vk = _view("q", q, sq, t, index), _view("k", k, sk, t, index)
    gq, gk = _view("d_q_out", d_q_out, sq, t, index), _view("d_k_out", d_k_out, sk, t, index)
    at, step, fr = _positions(rp, pos, freqs, sq, index)
    dq = _like(q, stream) if dq is None else dq
    dk = _like(k, stream) if dk is None else dk
    dwq = _floats(rp.d, index, stream) if dwq is None else dwq
    dwk = _floats(rp.d, index, stream) if dwk is None else dwk
    block = _block
    a = block.at
    try:
        _rotary_pack[6](block.buf, 0, *p, *vq, *vk, *gq, *gk, *_out("dq", dq, sq, t, index), *_out("dk", dk, sk, t, index))
    except _RANGE as e:
        raise _out_of_range(e) from None
    name = "mosaic_bsa_qk_norm_workspace_bytes"
    ws = _scratch(0 if ws is not None else int(getattr(_lib or lib(), name)(a)), name, index, ws, stream)
    _call("mosaic_bsa_qk_norm_bwd", index, stream, a, a + 40, a + 72, _flat("wq", wq, w, f32, index), _flat("wk", wk, w, f32, index),
          at, step, fr, a + 104, a + 136, a + 168, a + 200, _flat("dwq", dwq, w, f32, index), _flat("dwk", dwk, w, f32, index),
          ws.data_ptr(), ws.numel())
    return dq, dk, dwq, dwk


@dataclass(frozen=True)
class WindowParams:
    """Sliding-window attention: the row at position p sees the keys j <= p with p - j < window or j < sinks."""
    window: int
    sinks: int = 0
    scale: float = 0.0       # <= 0: 1/sqrt(d)
    rolling: bool = False    # decode: the cache keeps the sinks and, in turn, the last positions that fit behind them


def _window_params(wp, q, k):
    """(device, parameters, shape of k and v)"""
    index = _chk_seq(q, k)
    if q.dtype is torch.float32:
        raise ValueError("window attention takes bf16 or fp16 tensors")
    B, H, Nq, d = q.shape
    Hkv, Nk = k.shape[1], k.shape[2]
    flags = _STORAGE[q.dtype] | (FLAG_ROLLING if wp.rolling else 0)
    window = wp.window if wp.window < Nk or wp.rolling else Nk  # (Nk or more, whatever the number, is plain causal attention)
    return index, (B, H, Hkv, Nq, Nk, d, window, wp.sinks, wp.scale, flags), (B, Hkv, Nk, d)


def window_workspace_bytes(wp: WindowParams, q, k, op: int) -> int:
    return int(lib().mosaic_bsa_window_workspace_bytes(_params_block(_window_pack[0], _window_params(wp, q, k)[1]), op))


def _window_ws(at, op, index, ws, stream):
    name = "mosaic_bsa_window_workspace_bytes"
    return _scratch(0 if ws is not None else int(getattr(_lib or lib(), name)(at, op)), name, index, ws, stream)


def _rows_like(q, stream):
    """Contiguous fp32 [B, H, Nq] beside q (torch.empty takes a microsecond longer)."""
    if stream is not None:
        return _new(stream, _rows_like, q, None)
    B, H, N, _ = q.shape
    return torch.empty_strided((B, H, N), (H * N, N, 1), dtype=torch.float32, device=q.device)


def _len(name, t, B, index):
    return 0 if t is None else _flat(name, t, (B,), torch.int32, index)


def mosaic_bsa_window_fwd(wp: WindowParams, q, k, v, q_len=None, k_len=None, o=None, lse=None, ws=None, stream=None):
    """Forward of the sliding-window attention: q [B,H,Nq,d], k and v [B,Hkv,Nk,d]; the first q_len[b] and k_len[b] rows of a
    batch member exist (None: all), its queries are its last tokens.  Returns (o, lse)."""
    index, p, sk = _window_params(wp, q, k)
    t, sq = q.dtype, q.shape
    vq, vk, vv = _view("q", q, sq, t, index), _view("k", k, sk, t, index), _view("v", v, sk, t, index)
    o = _like(q, stream) if o is None else o
    lse = _rows_like(q, stream) if lse is None else lse
    block = _block
    a = block.at
    try:
        _window_pack[4](block.buf, 0, *p, *vq, *vk, *vv, *_out("o", o, sq, t, index))
    except _RANGE as e:
        raise _out_of_range(e) from None
    ws = _window_ws(a, OP_FWD, index, ws, stream)
    _call("mosaic_bsa_window_fwd", index, stream, a, a + 40, a + 72, a + 104, _len("q_len", q_len, sq[0], index),
          _len("k_len", k_len, sq[0], index), a + 136, _flat("lse", lse, sq[:3], torch.float32, index), ws.data_ptr(), ws.numel())
    return o, lse


def mosaic_bsa_window_bwd(wp: WindowParams, q, k, v, o, lse, d_o, q_len=None, k_len=None, dq=None, dk=None, dv=None, ws=None,
                          stream=None):
    """Backward of the sliding-window attention from the forward's inputs, its o and lse, and the gradient of o.
    Returns (dq, dk, dv)."""
    index, p, sk = _window_params(wp, q, k)
    t, sq = q.dtype, q.shape
    vq, vk, vv = _view("q", q, sq, t, index), _view("k", k, sk, t, index), _view("v", v, sk, t, index)
    vo, vd = _view("o", o, sq, t, index), _view("d_o", d_o, sq, t, index)
    dq = _like(q, stream) if dq is None else dq
    dk = _like(k, stream) if dk is None else dk
    dv = _like(v, stream) if dv is None else dv
    block = _block
    a = block.at
    try:
        _window_pack[8](block.buf, 0, *p, *vq, *vk, *vv, *vo, *vd, *_out("dq", dq, sq, t, index), *_out("dk", dk, sk, t, index),
                        *_out("dv", dv, sk, t, index))
    except _RANGE as e:
        raise _out_of_range(e) from None
    ws = _window_ws(a, OP_BWD, index, ws, stream)
    _call("mosaic_bsa_window_bwd", index, stream, a, a + 40, a + 72, a + 104, a + 136, _flat("lse", lse, sq[:3], torch.float32, index),
          a + 168, _len("q_len", q_len, sq[0], index), _len("k_len", k_len, sq[0], index), a + 200, a + 232, a + 264, ws.data_ptr(),
          ws.numel())
    return dq, dk, dv


def mosaic_bsa_window_decode(wp: WindowParams, q, k, v, k_len=None, o=None, lse=None, stream=None):
    """One new token per sequence: q [B,H,1,d] at position k_len[b] - 1 (None: the whole cache is filled), k and v [B,Hkv,Nk,d]
    with the token's own row in place.  `wp.rolling`: position j >= sinks lies in slot sinks + (j - sinks) % (Nk - sinks).
    Returns (o, lse)."""
    index, p, sk = _window_params(wp, q, k)
    t, sq = q.dtype, q.shape
    vq, vk, vv = _view("q", q, sq, t, index), _view("k", k, sk, t, index), _view("v", v, sk, t, index)
    o = _like(q, stream) if o is None else o
    lse = _rows_like(q, stream) if lse is None else lse
    block = _block
    a = block.at
    try:
        _window_pack[4](block.buf, 0, *p, *vq, *vk, *vv, *_out("o", o, sq, t, index))
    except _RANGE as e:
        raise _out_of_range(e) from None
    _call("mosaic_bsa_window_decode", index, stream, a, a + 40, a + 72, a + 104, _len("k_len", k_len, sq[0], index), a + 136,
          _flat("lse", lse, sq[:3], torch.float32, index))
    return o, lse
