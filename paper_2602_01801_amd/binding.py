"""ctypes front end of libfastar.so: argument marshalling only.

Every step of the path runs in the library's HIP kernels; PyTorch supplies device memory and the
stream.  Function names and argument meaning follow ``include/fastar.h``.  There is no fallback:
if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfastar.so")

F32, BF16 = 0, 1
OP_COMPRESS, OP_SELECT_SELF, OP_SELECT_CROSS, OP_SELECT_LSH, OP_SELECT_BUCKETS, OP_ATTN, OP_PAGED_ATTN, OP_PAGES = 1, 2, 3, 4, 5, 6, 7, 8
REP_LAST, REP_MEAN, REP_MEDOID = 0, 1, 2

_lib = None


class FastarError(RuntimeError):
    pass


class _CacheStruct(ctypes.Structure):
    _fields_ = [("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("code", ctypes.c_void_p), ("cnt", ctypes.c_void_p),
                ("stamp", ctypes.c_void_p), ("len", ctypes.c_void_p), ("H", ctypes.c_int32), ("C", ctypes.c_int32),
                ("d", ctypes.c_int32), ("r", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class _CodecStruct(ctypes.Structure):
    _fields_ = [("R", ctypes.c_void_p), ("qscale", ctypes.c_float), ("shift", ctypes.c_int32)]


class _RowsStruct(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("head", ctypes.c_int64), ("row", ctypes.c_int64)]


class _PagesStruct(ctypes.Structure):
    _fields_ = [("K8", ctypes.c_void_p), ("V8", ctypes.c_void_p), ("kscale", ctypes.c_void_p), ("vscale", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("P", ctypes.c_int32), ("d", ctypes.c_int32)]


class _RopeStruct(ctypes.Structure):
    _fields_ = [("qw", ctypes.c_void_p), ("kw", ctypes.c_void_p), ("freq", ctypes.c_void_p), ("axis", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("norm", ctypes.c_int32), ("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("n_axes", ctypes.c_int32)]


def lib() -> ctypes.CDLL:
    """Load libfastar.so (built in-tree by ``paper_2602_01801_amd.build``).  Fails loudly when absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FastarError(f"{LIB_PATH} is missing: run `python -m paper_2602_01801_amd.build` "
                              "(or __graft_entry__.build()) first; there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        L.fastar_init.restype = ctypes.c_int
        L.fastar_init.argtypes = []
        L.fastar_version.restype = ctypes.c_char_p
        L.fastar_strerror.restype = ctypes.c_char_p
        L.fastar_strerror.argtypes = [ctypes.c_int]
        L.fastar_workspace_bytes.restype = ctypes.c_size_t
        L.fastar_workspace_bytes.argtypes = [ctypes.c_int] * 8
        L.fastar_encode.restype = ctypes.c_int
        L.fastar_encode.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int,
                                    ctypes.POINTER(_CodecStruct), ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
        L.tempcache_compress.restype = ctypes.c_int
        L.tempcache_compress.argtypes = [ctypes.POINTER(_CacheStruct), ctypes.POINTER(_CodecStruct), ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
                                         ctypes.c_int, ctypes.c_int32, ctypes.c_int32, ctypes.c_int, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                         ctypes.c_int, ctypes.c_void_p]
        L.ann_cross_attn_fwd.restype = ctypes.c_int
        L.ann_cross_attn_fwd.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                         ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_float, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.ann_select_self.restype = ctypes.c_int
        L.ann_select_self.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int,
                                      ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                      ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.c_size_t, ctypes.c_void_p]
        L.ann_select_self_forced.restype = ctypes.c_int
        L.ann_select_self_forced.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p] + \
            [ctypes.c_int] * 9 + [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.ann_prompt_buckets.restype = ctypes.c_int
        L.ann_prompt_buckets.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p] + \
            [ctypes.c_int] * 4 + [ctypes.c_void_p, ctypes.c_void_p]
        L.ann_select_buckets.restype = ctypes.c_int
        L.ann_select_buckets.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p] + \
            [ctypes.c_int] * 9 + [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.fastar_encode_packed.restype = ctypes.c_int
        L.fastar_encode_packed.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int,
                                           ctypes.POINTER(_CodecStruct), ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
        L.ann_select_self_packed.restype = ctypes.c_int
        L.ann_select_self_packed.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p] + \
            [ctypes.c_int] * 10 + [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.ann_select_lsh_buckets.restype = ctypes.c_int
        L.ann_select_lsh_buckets.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p] + \
            [ctypes.c_int] * 11 + [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.ann_select_self_static.restype = ctypes.c_int
        L.ann_select_self_static.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int,
                                             ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                             ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.ann_select_cross.restype = ctypes.c_int
        L.ann_select_cross.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                       ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.sparse_attn_fwd.restype = ctypes.c_int
        L.sparse_attn_fwd.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                      ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                      ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.sparse_attn_fwd_ws.restype = ctypes.c_int
        L.sparse_attn_fwd_ws.argtypes = L.sparse_attn_fwd.argtypes[:-1] + [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.fastar_kv_to_fp8.restype = ctypes.c_int
        L.fastar_kv_to_fp8.argtypes = [ctypes.POINTER(_CacheStruct), ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p]
        L.sparse_attn_fwd_fp8.restype = ctypes.c_int
        L.sparse_attn_fwd_fp8.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.sparse_attn_fwd_fp8_ws.restype = ctypes.c_int
        L.sparse_attn_fwd_fp8_ws.argtypes = L.sparse_attn_fwd_fp8.argtypes[:-1] + [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.fastar_encode_sign.restype = ctypes.c_int
        L.fastar_encode_sign.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int, ctypes.c_void_p,
                                         ctypes.c_float, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
        L.ann_select_lsh.restype = ctypes.c_int
        L.ann_select_lsh.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p] + \
            [ctypes.c_int] * 7 + [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        rows = ctypes.POINTER(_RowsStruct)
        L.prompt_attn_fwd.restype = ctypes.c_int
        L.prompt_attn_fwd.argtypes = [rows, rows, rows, ctypes.c_void_p, ctypes.c_void_p] + [ctypes.c_int] * 8 + \
            [ctypes.c_float, rows, ctypes.c_void_p, ctypes.c_void_p]
        L.kv_pages_plan.restype = ctypes.c_int
        L.kv_pages_plan.argtypes = [ctypes.c_void_p] * 3 + [ctypes.c_int] * 2 + [ctypes.c_void_p] * 2 + [ctypes.c_int] * 3 + \
            [ctypes.c_void_p] * 6
        L.kv_pages_write.restype = ctypes.c_int
        L.kv_pages_write.argtypes = [ctypes.POINTER(_PagesStruct), rows, rows, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
                                     ctypes.c_void_p]
        L.paged_attn_fwd.restype = ctypes.c_int
        L.paged_attn_fwd.argtypes = [rows, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p] + [ctypes.c_int] * 4 + \
            [ctypes.POINTER(_PagesStruct), ctypes.c_int, ctypes.c_int, ctypes.c_float, rows, ctypes.c_void_p, ctypes.c_void_p,
             ctypes.c_size_t, ctypes.c_void_p]
        ptr, i32, pages, rope = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(_PagesStruct), ctypes.POINTER(_RopeStruct)
        L.qk_norm_rope.restype = i32
        L.qk_norm_rope.argtypes = [rows, rows, ptr, ptr, ptr] + [i32] * 6 + [rope, rows, rows, ptr]
        L.kv_pages_write_rope.restype = i32
        L.kv_pages_write_rope.argtypes = [pages, rows, rows, rows, i32, ptr, ptr, ptr, ptr, i32, i32, i32, rope, rows, ptr]
        L.kv_pages_fork.restype = i32
        L.kv_pages_fork.argtypes = [pages, ptr, ptr, ptr, i32, ptr, ptr, i32, i32, ptr, ptr, ptr, ptr, ptr, ptr]
        L.kv_pages_free.restype = i32
        L.kv_pages_free.argtypes = [ptr, ptr, ptr, i32, i32, ptr, ptr, i32, i32, ptr, ptr, ptr, ptr, ctypes.c_size_t, ptr]
        L.kv_pages_compact.restype = i32
        L.kv_pages_compact.argtypes = [pages, ptr, ptr, ptr, i32, i32] + [ptr] * 8 + [ctypes.c_size_t, ptr]
        L.fastar_probe_mfma_bf16.restype = ctypes.c_int
        L.fastar_probe_mfma_bf16.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.POINTER(ctypes.c_double), ctypes.c_void_p]
        L.fastar_probe_copy.restype = ctypes.c_int
        L.fastar_probe_copy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.fastar_probe_attn_route.restype = ctypes.c_int
        L.fastar_probe_attn_route.argtypes = [ctypes.c_int] * 6 + [ctypes.POINTER(ctypes.c_int)]
        L.fastar_debug_plan_wait.restype = ctypes.c_int
        L.fastar_debug_plan_wait.argtypes = [ctypes.c_int, ctypes.c_int]
        _lib = L
    return _lib


EXPORTS = ("fastar_init", "fastar_version", "fastar_strerror", "fastar_workspace_bytes", "fastar_encode", "tempcache_compress",
           "ann_cross_attn_fwd",
           "ann_select_self", "ann_select_self_forced", "ann_select_self_static", "ann_prompt_buckets", "ann_select_buckets", "fastar_encode_packed", "ann_select_self_packed", "ann_select_cross", "sparse_attn_fwd", "sparse_attn_fwd_ws", "fastar_kv_to_fp8",
           "sparse_attn_fwd_fp8", "sparse_attn_fwd_fp8_ws", "fastar_encode_sign", "ann_select_lsh", "ann_select_lsh_buckets",
           "prompt_attn_fwd", "kv_pages_plan", "kv_pages_write", "paged_attn_fwd", "qk_norm_rope", "kv_pages_write_rope", "kv_pages_fork", "kv_pages_free",
           "kv_pages_compact",
           "fastar_probe_mfma_bf16", "fastar_probe_copy", "fastar_probe_attn_route", "fastar_debug_plan_wait")


def init() -> None:
    """fastar_init: one-time kernel set-up for the current device (optional; needed before graph capture)."""
    _check(lib().fastar_init(), "fastar_init")


def _check(rc: int, what: str):
    if rc != 0:
        raise FastarError(f"{what}: {lib().fastar_strerror(rc).decode()} ({rc})")


# The handle of the current device's current stream.  torch.cuda.current_stream() builds a Stream object for it (3.0 us a call,
# as much as a launch; these two take 0.15); torch builds without them fall back to it.
_device_now = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None or _device_now is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device_now())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"dtype must be float32 or bfloat16, got {t.dtype}")


def _dev(t: torch.Tensor, dtype=None):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous device tensors")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    return t


# a function of its arguments alone: a look-up instead of a foreign call per checked workspace; typed, so that 2.0 is not 2
@functools.lru_cache(maxsize=256, typed=True)
def workspace_bytes(op: int, H: int, n_q: int, n_k: int, r: int = 32, BQ: int = 128, BK: int = 64,
                    n_rep: int = 4) -> int:
    return int(lib().fastar_workspace_bytes(op, H, n_q, n_k, r, BQ, BK, n_rep))


def _workspace(ws, nbytes: int, device):
    if ws is None:
        ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
    elif ws.get_device() != device.index or not ws.is_contiguous():   # a kernel writes through its address
        raise ValueError(f"the workspace must be a contiguous tensor on {device}, got one on {ws.device}")
    if ws.numel() * ws.element_size() < nbytes:
        raise FastarError("workspace too small")
    return ws


@dataclass
class Codec:
    """Definition of the ANN code: +-1 projection R [d,r] (device int8), quantiser scale, requantise shift."""
    R: torch.Tensor
    qscale: float
    shift: int

    def struct(self) -> _CodecStruct:
        _dev(self.R, torch.int8)
        return _CodecStruct(self.R.data_ptr(), float(self.qscale), int(self.shift))


@dataclass
class Cache:
    """Device buffers of the bounded per-head KV cache with multiplicities (capacity C slots per head)."""
    K: torch.Tensor      # [H,C,d]
    V: torch.Tensor      # [H,C,d]
    code: torch.Tensor   # [H,C,r] int8
    cnt: torch.Tensor    # [H,C] int32
    stamp: torch.Tensor  # [H,C] int32
    len: torch.Tensor    # [H] int32

    @classmethod
    def empty(cls, H: int, C: int, d: int, r: int, dtype: torch.dtype, device="cuda") -> "Cache":
        z = lambda *s, dt: torch.zeros(*s, dtype=dt, device=device)
        return cls(z(H, C, d, dt=dtype), z(H, C, d, dt=dtype), z(H, C, r, dt=torch.int8), z(H, C, dt=torch.int32),
                   z(H, C, dt=torch.int32), z(H, dt=torch.int32))

    @property
    def shape(self):
        H, C, d = self.K.shape
        return H, C, d, self.code.shape[2]

    def struct(self) -> _CacheStruct:
        H, C, d, r = self.shape
        for t in (self.K, self.V, self.code, self.cnt, self.stamp, self.len):
            if not t.is_cuda or not t.is_contiguous():   # _dev, without six calls of it
                _dev(t)
        return _CacheStruct(self.K.data_ptr(), self.V.data_ptr(), self.code.data_ptr(), self.cnt.data_ptr(),
                            self.stamp.data_ptr(), self.len.data_ptr(), H, C, d, r, _dtype_code(self.K))

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.K, self.V, self.code, self.cnt, self.stamp, self.len))


def encode(x: torch.Tensor, codec: Codec, out: torch.Tensor | None = None) -> torch.Tensor:
    """x [..., d] -> int8 codes [..., r]."""
    _dev(x)
    d, r = codec.R.shape
    n_vec = x.numel() // d
    if out is None:
        out = torch.empty(x.shape[:-1] + (r,), dtype=torch.int8, device=x.device)
    cs = codec.struct()
    _check(lib().fastar_encode(x.data_ptr(), _dtype_code(x), n_vec, d, ctypes.byref(cs), r, out.data_ptr(), _stream()),
           "fastar_encode")
    return out


def encode_packed(x: torch.Tensor, codec: Codec, bits: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """x [..., d] -> codes of `bits` (2, 4 or 8) bits per entry, packed: uint8 [..., r*bits/8]."""
    _dev(x)
    d, r = codec.R.shape
    n_vec = x.numel() // d
    if out is None:
        out = torch.empty(x.shape[:-1] + (r * bits // 8,), dtype=torch.uint8, device=x.device)
    cs = codec.struct()
    _check(lib().fastar_encode_packed(x.data_ptr(), _dtype_code(x), n_vec, d, ctypes.byref(cs), r, bits, out.data_ptr(),
                                      _stream()), "fastar_encode_packed")
    return out


def ann_select_self_packed(qcode, kcode, length, bits: int, BQ: int, n_rep: int, BK: int, n_sel: int, n_sink: int = 0,
                           n_local: int = 0, ws=None, out=None):
    """AnnSA on packed codes (uint8 [H,n,r*bits/8]): the selection ann_select_self makes on the unpacked entries."""
    _dev(qcode, torch.uint8)
    _dev(kcode, torch.uint8)
    _dev(length, torch.int32)
    H, n_q, rb = qcode.shape
    r = rb * 8 // bits
    C = kcode.shape[1]
    n_qb = (n_q + BQ - 1) // BQ
    ws = _workspace(ws, workspace_bytes(OP_SELECT_SELF, H, n_q, C, r, BQ, BK, n_rep), qcode.device)
    if out is None:
        out = (torch.empty((H, n_qb, n_sel), dtype=torch.int32, device=qcode.device),
               torch.empty((H, n_qb), dtype=torch.int32, device=qcode.device))
    sel, nsel = out
    _check(lib().ann_select_self_packed(qcode.data_ptr(), n_q, kcode.data_ptr(), length.data_ptr(), H, C, r, bits, BQ,
                                        n_rep, BK, n_sel, n_sink, n_local, sel.data_ptr(), nsel.data_ptr(), ws.data_ptr(),
                                        ws.numel() * ws.element_size(), _stream()), "ann_select_self_packed")
    return sel, nsel


def tempcache_compress(cache: Cache, codec: Codec, K_new, V_new, P_new=None, cand=None, metric: int = 0,
                       tau2_q16: int = 53084, frame_id: int = 0, rep_mode: int = 0, ws=None, out=None,
                       ws_persistent: bool = False):
    """Merge one frame into ``cache`` in place.  Returns (merge_map [H,n] int32, merged [H,n] uint8, stats [H,8]).
    rep_mode: REP_LAST (0) keeps the last key of a merged group, REP_MEAN (1) its multiplicity-weighted mean.
    ws_persistent: ``ws`` was zero-filled once and has since been written only by calls on this cache (one launch less)."""
    if ws_persistent and ws is None:
        raise ValueError("ws_persistent needs the caller's own workspace")
    H, C, d, r = cache.shape
    _dev(K_new, cache.K.dtype)
    _dev(V_new, cache.K.dtype)
    n_new = K_new.shape[1]
    if P_new is not None:
        _dev(P_new, cache.K.dtype)
    n_cand = 0
    if cand is not None:
        _dev(cand, torch.int32)
        n_cand = cand.shape[1]
    ws = _workspace(ws, workspace_bytes(OP_COMPRESS, H, n_new, C, r), K_new.device)
    if out is None:
        out = (torch.empty((H, n_new), dtype=torch.int32, device=K_new.device),
               torch.empty((H, n_new), dtype=torch.uint8, device=K_new.device),
               torch.empty((H, 8), dtype=torch.int32, device=K_new.device))
    merge_map, merged, stats = out
    cs, ks = cache.struct(), codec.struct()
    _check(lib().tempcache_compress(ctypes.byref(cs), ctypes.byref(ks), K_new.data_ptr(), V_new.data_ptr(),
                                    _ptr(P_new), n_new, _ptr(cand), n_cand, metric, tau2_q16, frame_id,
                                    int(rep_mode), merge_map.data_ptr(), merged.data_ptr(), stats.data_ptr(), ws.data_ptr(),
                                    ws.numel() * ws.element_size(), 1 if ws_persistent else 0, _stream()),
           "tempcache_compress")
    return merge_map, merged, stats


def ann_select_self(qcode, kcode, length, BQ: int, n_rep: int, BK: int, n_sel: int, ws=None, out=None, n_sink: int = 0,
                    n_local: int = 0):
    """AnnSA: (sel [H,n_qb,n_sel] int32 ascending / -1 padded, nsel [H,n_qb] int32).  n_sink / n_local > 0 calls
    ann_select_self_forced (first / last live key blocks always selected)."""
    _dev(qcode, torch.int8)
    _dev(kcode, torch.int8)
    _dev(length, torch.int32)
    H, n_q, r = qcode.shape
    C = kcode.shape[1]
    n_qb = (n_q + BQ - 1) // BQ
    ws = _workspace(ws, workspace_bytes(OP_SELECT_SELF, H, n_q, C, r, BQ, BK, n_rep), qcode.device)
    if out is None:
        out = (torch.empty((H, n_qb, n_sel), dtype=torch.int32, device=qcode.device),
               torch.empty((H, n_qb), dtype=torch.int32, device=qcode.device))
    sel, nsel = out
    if n_sink or n_local:
        _check(lib().ann_select_self_forced(qcode.data_ptr(), n_q, kcode.data_ptr(), length.data_ptr(), H, C, r, BQ, n_rep,
                                            BK, n_sel, n_sink, n_local, sel.data_ptr(), nsel.data_ptr(), ws.data_ptr(),
                                            ws.numel() * ws.element_size(), _stream()), "ann_select_self_forced")
        return sel, nsel
    _check(lib().ann_select_self(qcode.data_ptr(), n_q, kcode.data_ptr(), length.data_ptr(), H, C, r, BQ, n_rep, BK,
                                 n_sel, sel.data_ptr(), nsel.data_ptr(), ws.data_ptr(),
                                 ws.numel() * ws.element_size(), _stream()), "ann_select_self")
    return sel, nsel


def ann_select_self_static(qcode, kcode, length, BQ: int, n_rep: int, BK: int, n_sel: int, out):
    """AnnSA on the library's static scratch: the call allocates nothing, so the outputs (sel, nsel) must be given."""
    _dev(qcode, torch.int8)
    _dev(kcode, torch.int8)
    _dev(length, torch.int32)
    H, n_q, r = qcode.shape
    C = kcode.shape[1]
    sel, nsel = out
    _dev(sel, torch.int32)
    _dev(nsel, torch.int32)
    n_qb = (n_q + BQ - 1) // BQ
    if tuple(sel.shape) != (H, n_qb, n_sel) or tuple(nsel.shape) != (H, n_qb):
        raise ValueError("out must be (sel [H,n_qb,n_sel], nsel [H,n_qb])")
    _check(lib().ann_select_self_static(qcode.data_ptr(), n_q, kcode.data_ptr(), length.data_ptr(), H, C, r, BQ, n_rep,
                                        BK, n_sel, sel.data_ptr(), nsel.data_ptr(), _stream()), "ann_select_self_static")
    return sel, nsel


def prompt_buckets(code, pcode, m: int = 1, idx=None, out=None):
    """The m nearest prompt tokens of every code row: bucket [H,C,m] int32.  idx [H,n] int32 names the rows to assign
    (the others keep what `out` holds); without it every row is assigned."""
    _dev(code, torch.int8)
    _dev(pcode, torch.int8)
    H, C, r = code.shape
    n_p = pcode.shape[1]
    if out is None:
        out = torch.full((H, C, m), -1, dtype=torch.int32, device=code.device)
    if idx is not None:
        _dev(idx, torch.int32)
    n = C if idx is None else idx.shape[1]
    _check(lib().ann_prompt_buckets(code.data_ptr(), C, idx.data_ptr() if idx is not None else None, n, pcode.data_ptr(),
                                    n_p, H, r, m, out.data_ptr(), _stream()), "ann_prompt_buckets")
    return out


def ann_select_buckets(qbucket, kbucket, length, n_p: int, BQ: int, BK: int, n_sel: int, n_sink: int = 0, n_local: int = 0,
                       ws=None, out=None):
    """AnnSA on prompt-induced buckets: (sel [H,n_qb,n_sel] int32 ascending / -1 padded, nsel [H,n_qb] int32)."""
    _dev(qbucket, torch.int32)
    _dev(kbucket, torch.int32)
    _dev(length, torch.int32)
    H, n_q, m = qbucket.shape
    C = kbucket.shape[1]
    n_qb = (n_q + BQ - 1) // BQ
    ws = _workspace(ws, workspace_bytes(OP_SELECT_BUCKETS, H, n_q, C, n_p, BQ, BK, 0), qbucket.device)
    if out is None:
        out = (torch.empty((H, n_qb, n_sel), dtype=torch.int32, device=qbucket.device),
               torch.empty((H, n_qb), dtype=torch.int32, device=qbucket.device))
    sel, nsel = out
    _check(lib().ann_select_buckets(qbucket.data_ptr(), n_q, kbucket.data_ptr(), length.data_ptr(), H, C, m, n_p, BQ, BK,
                                    n_sel, n_sink, n_local, sel.data_ptr(), nsel.data_ptr(), ws.data_ptr(),
                                    ws.numel() * ws.element_size(), _stream()), "ann_select_buckets")
    return sel, nsel


def ann_select_cross(qcode, pcode, BQ: int, n_sel: int, ws=None, out=None):
    """AnnCA: (sel [H,n_qb,n_sel] prompt-token ids ascending / -1 padded, nsel [H,n_qb])."""
    _dev(qcode, torch.int8)
    _dev(pcode, torch.int8)
    H, n_q, r = qcode.shape
    n_p = pcode.shape[1]
    n_qb = (n_q + BQ - 1) // BQ
    ws = _workspace(ws, workspace_bytes(OP_SELECT_CROSS, H, n_q, n_p, r, BQ), qcode.device)
    if out is None:
        out = (torch.empty((H, n_qb, n_sel), dtype=torch.int32, device=qcode.device),
               torch.empty((H, n_qb), dtype=torch.int32, device=qcode.device))
    sel, nsel = out
    _check(lib().ann_select_cross(qcode.data_ptr(), n_q, pcode.data_ptr(), n_p, H, r, BQ, n_sel, sel.data_ptr(),
                                  nsel.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _stream()),
           "ann_select_cross")
    return sel, nsel


def encode_sign(x: torch.Tensor, R: torch.Tensor, qscale: float, out: torch.Tensor | None = None) -> torch.Tensor:
    """x [..., d], R [d, n_bits] int8 (+-1) -> sign codes [..., n_bits/32] as int32 words (bit patterns)."""
    _dev(x)
    _dev(R, torch.int8)
    d, n_bits = R.shape
    if x.shape[-1] != d or not x.is_contiguous() or not R.is_contiguous():
        raise ValueError("encode_sign: x must be contiguous [..., d] and R contiguous [d, n_bits]")
    n_vec = x.numel() // d
    if out is None:
        out = torch.empty(x.shape[:-1] + (n_bits // 32,), dtype=torch.int32, device=x.device)
    _check(lib().fastar_encode_sign(x.data_ptr(), _dtype_code(x), n_vec, d, R.data_ptr(), float(qscale), n_bits,
                                    out.data_ptr(), _stream()), "fastar_encode_sign")
    return out


def ann_select_lsh(qbits, kbits, length, BQ: int, n_rep: int, BK: int, n_sel: int, ws=None, out=None):
    """Selection on sign codes: (sel [H,n_qb,n_sel] int32 ascending / -1 padded, nsel [H,n_qb] int32)."""
    _dev(qbits, torch.int32)
    _dev(kbits, torch.int32)
    _dev(length, torch.int32)
    H, n_q, W = qbits.shape
    C = kbits.shape[1]
    n_qb = (n_q + BQ - 1) // BQ
    ws = _workspace(ws, workspace_bytes(OP_SELECT_LSH, H, n_q, C, 32 * W, BQ, BK, n_rep), qbits.device)
    if out is None:
        out = (torch.empty((H, n_qb, n_sel), dtype=torch.int32, device=qbits.device),
               torch.empty((H, n_qb), dtype=torch.int32, device=qbits.device))
    sel, nsel = out
    _check(lib().ann_select_lsh(qbits.data_ptr(), n_q, kbits.data_ptr(), length.data_ptr(), H, C, 32 * W, BQ, n_rep,
                                BK, n_sel, sel.data_ptr(), nsel.data_ptr(), ws.data_ptr(),
                                ws.numel() * ws.element_size(), _stream()), "ann_select_lsh")
    return sel, nsel


def ann_select_lsh_buckets(qbits, kbits, length, band_bits: int, radius: int, BQ: int, n_rep: int, BK: int, n_sel: int,
                           n_sink: int = 0, n_local: int = 0, ws=None, out=None):
    """Hash-table form of ann_select_lsh (bands = tables, buckets at most `radius` bits apart collide)."""
    _dev(qbits, torch.int32)
    _dev(kbits, torch.int32)
    _dev(length, torch.int32)
    H, n_q, W = qbits.shape
    C = kbits.shape[1]
    n_qb = (n_q + BQ - 1) // BQ
    ws = _workspace(ws, workspace_bytes(OP_SELECT_LSH, H, n_q, C, 32 * W, BQ, BK, n_rep), qbits.device)
    if out is None:
        out = (torch.empty((H, n_qb, n_sel), dtype=torch.int32, device=qbits.device),
               torch.empty((H, n_qb), dtype=torch.int32, device=qbits.device))
    sel, nsel = out
    _check(lib().ann_select_lsh_buckets(qbits.data_ptr(), n_q, kbits.data_ptr(), length.data_ptr(), H, C, 32 * W,
                                        band_bits, radius, BQ, n_rep, BK, n_sel, n_sink, n_local, sel.data_ptr(),
                                        nsel.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _stream()),
           "ann_select_lsh_buckets")
    return sel, nsel


def ann_cross_attn_fwd(Q, qcode, Kp, Vp, pcode, BQ: int, n_sel: int, scale: float, out=None):
    """AnnCA selection and the attention over it in one launch.  Returns (sel [H,n_qb,n_sel], nsel [H,n_qb], O)."""
    _dev(Q)
    _dev(Kp, Q.dtype)
    _dev(Vp, Q.dtype)
    _dev(qcode, torch.int8)
    _dev(pcode, torch.int8)
    H, n_q, d = Q.shape
    n_p, r = pcode.shape[1], pcode.shape[2]
    n_qb = (n_q + BQ - 1) // BQ
    if out is None:
        out = (torch.empty((H, n_qb, n_sel), dtype=torch.int32, device=Q.device),
               torch.empty((H, n_qb), dtype=torch.int32, device=Q.device), torch.empty_like(Q))
    sel, nsel, O = out
    _check(lib().ann_cross_attn_fwd(Q.data_ptr(), qcode.data_ptr(), n_q, Kp.data_ptr(), Vp.data_ptr(), pcode.data_ptr(),
                                    n_p, H, d, _dtype_code(Q), r, BQ, n_sel, float(scale), sel.data_ptr(),
                                    nsel.data_ptr(), O.data_ptr(), _stream()), "ann_cross_attn_fwd")
    return sel, nsel, O


def sparse_attn_fwd(Q, K, V, cnt, length, sel, nsel, BQ: int, BK: int, scale: float, out=None, want_lse: bool = True,
                    ws=None):
    """Block-sparse attention.  Returns (O [H,n_q,d] in Q's dtype, lse [H,n_q] float32 or None).
    ws: uint8 device workspace of workspace_bytes(OP_ATTN, ...) -> sparse_attn_fwd_ws (several workgroups per query block
    where that pays; calls that may be in flight at the same time need a workspace each)."""
    _dev(Q)
    _dev(K, Q.dtype)
    _dev(V, Q.dtype)
    _dev(length, torch.int32)
    _dev(sel, torch.int32)
    _dev(nsel, torch.int32)
    if cnt is not None:
        _dev(cnt, torch.int32)
    H, n_q, d = Q.shape
    C = K.shape[1]
    n_sel = sel.shape[2]
    if out is None:
        out = (torch.empty_like(Q), torch.empty((H, n_q), dtype=torch.float32, device=Q.device) if want_lse else None)
    O, lse = out
    if ws is not None:
        _dev(ws, torch.uint8)
        _check(lib().sparse_attn_fwd_ws(Q.data_ptr(), n_q, K.data_ptr(), V.data_ptr(), _ptr(cnt), length.data_ptr(), H, C,
                                        d, _dtype_code(Q), sel.data_ptr(), nsel.data_ptr(), BQ, BK, n_sel, float(scale),
                                        O.data_ptr(), _ptr(lse), ws.data_ptr(), ws.numel(), _stream()),
               "sparse_attn_fwd_ws")
        return O, lse
    _check(lib().sparse_attn_fwd(Q.data_ptr(), n_q, K.data_ptr(), V.data_ptr(), _ptr(cnt), length.data_ptr(), H, C, d,
                                 _dtype_code(Q), sel.data_ptr(), nsel.data_ptr(), BQ, BK, n_sel, float(scale),
                                 O.data_ptr(), _ptr(lse), _stream()), "sparse_attn_fwd")
    return O, lse


def kv8_empty(H: int, C: int, d: int = 128, device="cuda"):
    """Zero-filled 8-bit copy of a cache of capacity C: (K8 [H,Cp,d], V8T [H,Cp/64,d,64]) uint8, Cp = C rounded up to 64."""
    n_blk = (C + 63) // 64
    return (torch.zeros((H, n_blk * 64, d), dtype=torch.uint8, device=device),
            torch.zeros((H, n_blk, d, 64), dtype=torch.uint8, device=device))


def kv_to_fp8(cache: Cache, K8: torch.Tensor, V8T: torch.Tensor, stamp_lo: int = -2 ** 31) -> None:
    """fastar_kv_to_fp8: rewrite the blocks of the 8-bit copy that hold a live slot with stamp >= stamp_lo."""
    H, C, d, _ = cache.shape
    n_blk = (C + 63) // 64
    _dev(K8, torch.uint8)
    _dev(V8T, torch.uint8)
    if tuple(K8.shape) != (H, n_blk * 64, d) or tuple(V8T.shape) != (H, n_blk, d, 64):
        raise ValueError("K8 must be [H,Cp,d] and V8T [H,Cp/64,d,64] with Cp = C rounded up to a multiple of 64")
    cs = cache.struct()
    _check(lib().fastar_kv_to_fp8(ctypes.byref(cs), int(stamp_lo), K8.data_ptr(), V8T.data_ptr(), _stream()),
           "fastar_kv_to_fp8")


def sparse_attn_fwd_fp8(Q, K8, V8T, cnt, length, C: int, sel, nsel, BQ: int, BK: int, scale: float, out=None,
                        want_lse: bool = True, ws=None):
    """Block-sparse attention over the 8-bit cache copy.  Returns (O [H,n_q,d] bf16, lse [H,n_q] float32 or None).
    ws: workspace of workspace_bytes(OP_ATTN, ...) -> sparse_attn_fwd_fp8_ws (as for sparse_attn_fwd)."""
    _dev(Q, torch.bfloat16)
    _dev(K8, torch.uint8)
    _dev(V8T, torch.uint8)
    _dev(length, torch.int32)
    _dev(sel, torch.int32)
    _dev(nsel, torch.int32)
    if cnt is not None:
        _dev(cnt, torch.int32)
    H, n_q, d = Q.shape
    n_blk = (C + 63) // 64
    if tuple(K8.shape) != (H, n_blk * 64, d) or tuple(V8T.shape) != (H, n_blk, d, 64):
        raise ValueError("K8 must be [H,Cp,d] and V8T [H,Cp/64,d,64] with Cp = C rounded up to a multiple of 64")
    n_sel = sel.shape[2]
    if out is None:
        out = (torch.empty_like(Q), torch.empty((H, n_q), dtype=torch.float32, device=Q.device) if want_lse else None)
    O, lse = out
    if ws is not None:
        _dev(ws, torch.uint8)
        _check(lib().sparse_attn_fwd_fp8_ws(Q.data_ptr(), n_q, K8.data_ptr(), V8T.data_ptr(), _ptr(cnt), length.data_ptr(),
                                            H, C, d, sel.data_ptr(), nsel.data_ptr(), BQ, BK, n_sel, float(scale),
                                            O.data_ptr(), _ptr(lse), ws.data_ptr(), ws.numel(), _stream()),
               "sparse_attn_fwd_fp8_ws")
        return O, lse
    _check(lib().sparse_attn_fwd_fp8(Q.data_ptr(), n_q, K8.data_ptr(), V8T.data_ptr(), _ptr(cnt), length.data_ptr(), H, C,
                                     d, sel.data_ptr(), nsel.data_ptr(), BQ, BK, n_sel, float(scale), O.data_ptr(),
                                     _ptr(lse), _stream()), "sparse_attn_fwd_fp8")
    return O, lse


# ---------------------------------------------------------------------------------------------- several requests at a time


def _here() -> int:
    """The device whose current stream a call is launched on."""
    return torch.cuda.current_device() if _device_now is None else _device_now()


# The checks below are what a call costs on the host, next to the foreign call itself: one condition each where all is well.
def _rows(t: torch.Tensor, H: int, n: int, d: int, dtype, dev: int) -> _RowsStruct:
    """A view [H, n, d] of any head and row strides."""
    if t.dtype is not dtype or t.shape != (H, n, d) or t.get_device() != dev:
        if t.dtype != dtype:
            raise TypeError(f"expected {dtype}, got {t.dtype}")
        raise ValueError(f"expected a tensor [{H}, {n}, {d}] on the current device, got {tuple(t.shape)} on {t.device}")
    head, row, one = t.stride()
    if one != 1:
        raise ValueError("rows must be contiguous")
    return _RowsStruct(t.data_ptr(), head, row)


def _ints(t: torch.Tensor, n: int, dev: int) -> int:
    """n contiguous int32 numbers."""
    if t.dtype is not torch.int32 or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        _dev(t, torch.int32)
        raise ValueError(f"expected {n} numbers on the current device, got {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _lse_out(lse, Hq: int, n: int, dev: int):
    if lse is None:
        return None
    if lse.shape != (Hq, n) or lse.dtype is not torch.float32 or lse.get_device() != dev or not lse.is_contiguous():
        _dev(lse, torch.float32)
        raise ValueError(f"lse must be [{Hq}, {n}] on the current device, got {tuple(lse.shape)} on {lse.device}")
    return lse.data_ptr()


def _grouped(Q, Hkv: int):
    if Q.dim() != 3:
        raise ValueError("Q must be [Hq, n, d]")
    Hq, n, d = Q.shape
    if Hkv <= 0 or Hq % Hkv:
        raise ValueError(f"{Hq} query heads cannot share {Hkv} key heads")
    return Hq, n, d


def prompt_attn_fwd(Q, K, V, cu_q, cu_k=None, causal: bool = True, scale: float | None = None, out=None, want_lse: bool = True):
    """Attention over whole packed prompts.  Q [Hq,n_q,d], K, V [Hkv,n_k,d]: views of any head and row strides; cu_q, cu_k
    [B+1] int32 (cu_k None: cu_q); scale None: d ** -0.5.  Returns (O [Hq,n_q,d] in Q's dtype, lse [Hq,n_q] or None); rows
    outside of every sequence are not written."""
    Hq, n_q, d = _grouped(Q, K.shape[0])
    Hkv, n_k = K.shape[0], K.shape[1]
    dt, code, dev = Q.dtype, _dtype_code(Q), _here()
    B = cu_q.numel() - 1
    if out is None:
        out = (torch.empty_like(Q), torch.empty((Hq, n_q), dtype=torch.float32, device=Q.device) if want_lse else None)
    O, lse = out
    _check(lib().prompt_attn_fwd(_rows(Q, Hq, n_q, d, dt, dev), _rows(K, Hkv, n_k, d, dt, dev), _rows(V, Hkv, n_k, d, dt, dev),
                                 _ints(cu_q, B + 1, dev), None if cu_k is None else _ints(cu_k, B + 1, dev), B, n_q, n_k, Hq, Hkv, d,
                                 code, 1 if causal else 0, d ** -0.5 if scale is None else float(scale), _rows(O, Hq, n_q, d, dt, dev),
                                 _lse_out(lse, Hq, n_q, dev), _stream()), "prompt_attn_fwd")
    return O, lse


@dataclass(frozen=True)
class Pages:
    """Device buffers of a paged cache of E4M3 codes with a scale per page and head (fastar_pages); checked once, when it is made."""
    K8: torch.Tensor      # [n_pages, Hkv, P/16, d/16, 16 tokens, 16 coordinates] uint8
    kscale: torch.Tensor  # [n_pages, Hkv] float32
    V8: torch.Tensor      # [n_pages, Hkv, P/16, d/16, 16 coordinates, 16 tokens] uint8
    vscale: torch.Tensor  # [n_pages, Hkv] float32

    @classmethod
    def empty(cls, n_pages: int, Hkv: int, P: int, d: int, device="cuda") -> "Pages":
        code = lambda: torch.zeros((n_pages, Hkv, P // 16, d // 16, 16, 16), dtype=torch.uint8, device=device)
        one = lambda: torch.ones((n_pages, Hkv), dtype=torch.float32, device=device)
        return cls(code(), one(), code(), one())

    def __post_init__(self):
        shape = tuple(self.K8.shape)
        if len(shape) != 6 or shape[4:] != (16, 16):
            raise ValueError("K8 and V8 must be [n_pages, Hkv, P/16, d/16, 16, 16], kscale and vscale [n_pages, Hkv]")
        for t, want, dtype in ((self.K8, shape, torch.uint8), (self.V8, shape, torch.uint8), (self.kscale, shape[:2], torch.float32),
                               (self.vscale, shape[:2], torch.float32)):
            if tuple(_dev(t, dtype).shape) != want or t.device != self.K8.device:
                raise ValueError("K8 and V8 must be [n_pages, Hkv, P/16, d/16, 16, 16], kscale and vscale [n_pages, Hkv], on one device")
        object.__setattr__(self, "shape", (shape[0], shape[1], 16 * shape[2], 16 * shape[3]))   # (n_pages, Hkv, P, d)

    def struct(self, dev: int) -> _PagesStruct:
        if self.K8.get_device() != dev:
            raise ValueError("the pages are not on the current device")
        return _PagesStruct(self.K8.data_ptr(), self.V8.data_ptr(), self.kscale.data_ptr(), self.vscale.data_ptr(), *self.shape)

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.K8, self.V8, self.kscale, self.vscale))


def kv_pages_plan(n_new, length, table, pool, pool_n, P: int, n_tok: int, out=None):
    """Block tables and slot maps of the next step: n_new, length [B] int32, table [B,max_pages] and pool [n_pages] int32
    (updated in place), pool_n [1] int32, n_tok rows for new tokens.  Returns (length after, pool_n after, cu [B+1],
    slot [n_tok], status [B]), all int32; out may name `length` and `pool_n` themselves for the first two.  Slots behind the
    last new token are -1, in an array of the caller's as they were: it sets them to -1 where a step has fewer tokens than n_tok."""
    B, max_pages = table.shape
    n_pages, dev = pool.numel(), _here()
    if out is None:
        i = lambda *n: torch.empty(n, dtype=torch.int32, device=table.device)
        out = (i(B), i(1), i(B + 1), torch.full((n_tok,), -1, dtype=torch.int32, device=table.device), i(B))
    after, free, cu, slot, status = out
    _check(lib().kv_pages_plan(_ints(n_new, B, dev), _ints(length, B, dev), _ints(table, B * max_pages, dev), B, max_pages,
                               _ints(pool, n_pages, dev), _ints(pool_n, 1, dev), n_pages, P, n_tok, _ints(after, B, dev),
                               _ints(free, 1, dev), _ints(cu, B + 1, dev), _ints(slot, n_tok, dev), _ints(status, B, dev), _stream()),
           "kv_pages_plan")
    return out


def kv_pages_write(pages: Pages, slot, K_new, V_new) -> None:
    """New keys and values [Hkv,n,d] (views of any head and row strides) into the pages' slots [n] int32 (kv_pages_plan)."""
    dev = _here()
    ps = pages.struct(dev)
    n, dt, code = slot.numel(), K_new.dtype, _dtype_code(K_new)
    _check(lib().kv_pages_write(ps, _rows(K_new, ps.Hkv, n, ps.d, dt, dev), _rows(V_new, ps.Hkv, n, ps.d, dt, dev), code,
                                _ints(slot, n, dev), n, _stream()), "kv_pages_write")


def paged_attn_fwd(Q, cu_q, length, table, pages: Pages, causal: bool = True, scale: float | None = None, out=None,
                   want_lse: bool = True, ws=None):
    """Attention of packed queries Q [Hq,n,d] bf16 (a view of any head and row strides) over the pages of their sequences:
    cu_q [B+1], length [B] and table [B,max_pages] int32.  Returns (O [Hq,n,d], lse [Hq,n] or None).
    ws: workspace of workspace_bytes(OP_PAGED_ATTN, ...); calls that may be in flight at the same time need one each."""
    dev = _here()
    ps = pages.struct(dev)
    Hq, n, d = _grouped(Q, ps.Hkv)
    dt, code = Q.dtype, _dtype_code(Q)
    B, max_pages = table.shape
    ws = _workspace(ws, workspace_bytes(OP_PAGED_ATTN, Hq, n, 0), Q.device)
    if out is None:
        out = (torch.empty_like(Q), torch.empty((Hq, n), dtype=torch.float32, device=Q.device) if want_lse else None)
    O, lse = out
    _check(lib().paged_attn_fwd(_rows(Q, Hq, n, ps.d, dt, dev), _ints(cu_q, B + 1, dev), _ints(length, B, dev),
                                _ints(table, B * max_pages, dev), B, max_pages, n, Hq, ps, code, 1 if causal else 0,
                                d ** -0.5 if scale is None else float(scale), _rows(O, Hq, n, ps.d, dt, dev),
                                _lse_out(lse, Hq, n, dev), ws.data_ptr(), ws.numel() * ws.element_size(), _stream()), "paged_attn_fwd")
    return O, lse


@dataclass(frozen=True)
class Rope:
    """Norm and rotation of queries and keys (fastar_rope); checked once, when it is made."""
    freq: torch.Tensor | None                # [rot/2] float64: radians per position of every pair; None: no rotation
    axis: torch.Tensor | None = None         # [rot/2] int32: row of the positions that a pair goes by; None: row 0
    n_axes: int = 1                          # rows of the positions
    norm: bool = True                        # root mean square per head
    q_weight: torch.Tensor | None = None     # [d] float32; None: ones
    k_weight: torch.Tensor | None = None
    eps: float = 1e-6
    interleaved: bool = False                # pairs (2i, 2i+1) instead of (i, i + rot/2)

    def __post_init__(self):
        rot = 0 if self.freq is None else 2 * _dev(self.freq, torch.float64).numel()
        if self.axis is not None and _dev(self.axis, torch.int32).numel() * 2 != rot:
            raise ValueError("axis must name one row of the positions per pair")
        d = {_dev(w, torch.float32).numel() for w in (self.q_weight, self.k_weight) if w is not None}
        if len({t.device for t in (self.freq, self.axis, self.q_weight, self.k_weight) if t is not None}) > 1 or len(d) > 1:
            raise ValueError("frequencies, axes and weights must be on one device, and the weights as many as a head's coordinates")
        device = next((t.get_device() for t in (self.freq, self.axis, self.q_weight, self.k_weight) if t is not None), None)
        for name, value in (("rot", rot), ("d", d.pop() if d else None), ("device", device), (
                "_struct", _RopeStruct(_ptr(self.q_weight), _ptr(self.k_weight), _ptr(self.freq), _ptr(self.axis), float(self.eps),
                                       int(self.norm), rot, int(self.interleaved), self.n_axes))):
            object.__setattr__(self, name, value)

    def struct(self, d: int, dev: int) -> _RopeStruct:
        if (self.d is not None and self.d != d) or (self.device is not None and self.device != dev):
            raise ValueError(f"expected weights of {d} coordinates on the current device, got {self.d} on {self.device}")
        return self._struct


def _positions(rope: Rope, pos, cu, length, n: int, dev: int):
    """Pointers of pos, cu and length, and the number of sequences."""
    if pos is not None and pos.shape != (rope.n_axes, n):
        raise ValueError(f"pos must be [{rope.n_axes}, {n}], got {tuple(pos.shape)}")
    if cu is None:
        return None if pos is None else _ints(pos, rope.n_axes * n, dev), None, None, 0
    B = cu.numel() - 1
    return (None if pos is None else _ints(pos, rope.n_axes * n, dev), _ints(cu, B + 1, dev),
            None if length is None else _ints(length, B, dev), B)


def qk_norm_rope(Q, K, rope: Rope, pos=None, cu=None, length=None, out=None):
    """Queries [Hq,n,d] and keys [Hkv,n,d] (views of any head and row strides; either may be None) normed per head and rotated by
    their positions pos [n_axes,n] int32.  pos None: row i of the a rows of a sequence (cu [B+1] int32) is at length - a + i (length
    [B] int32).  Returns (Q, K) in their type, in `out`, which may be (Q, K) itself; rows outside of every sequence are not written."""
    some = Q if Q is not None else K
    if some is None or some.dim() != 3:
        raise ValueError("Q and K must be [heads, n, d]")
    n, d, dt, code, dev = some.shape[1], some.shape[2], some.dtype, _dtype_code(some), _here()
    if out is None:
        out = tuple(None if x is None else torch.empty_like(x) for x in (Q, K))
    Hq, Hkv = (0 if x is None else x.shape[0] for x in (Q, K))
    q, qo, k, ko = (None if x is None else _rows(x, H, n, d, dt, dev) for x, H in ((Q, Hq), (out[0], Hq), (K, Hkv), (out[1], Hkv)))
    pos, cu, length, B = _positions(rope, pos, cu, length, n, dev)
    _check(lib().qk_norm_rope(q, k, pos, cu, length, B, n, Hq, Hkv, d, code, rope.struct(d, dev), qo, ko, _stream()), "qk_norm_rope")
    return out


def kv_pages_write_rope(pages: Pages, slot, Q, K_new, V_new, rope: Rope, pos=None, cu=None, length=None, out=None):
    """qk_norm_rope of Q [Hq,n,d] (None: keys only) and K_new [Hkv,n,d], and kv_pages_write of those keys and V_new into the slots [n].
    Returns Q normed and rotated, in `out`, which may be Q itself."""
    dev = _here()
    ps = pages.struct(dev)
    n, dt, code = slot.numel(), K_new.dtype, _dtype_code(K_new)
    if Q is not None and out is None:
        out = torch.empty_like(Q)
    Hq = 0 if Q is None else Q.shape[0]
    q, qo = (None if Q is None else _rows(x, Hq, n, ps.d, dt, dev) for x in (Q, out))
    pos, cu, length, B = _positions(rope, pos, cu, length, n, dev)
    _check(lib().kv_pages_write_rope(ps, q, _rows(K_new, ps.Hkv, n, ps.d, dt, dev), _rows(V_new, ps.Hkv, n, ps.d, dt, dev), code,
                                     _ints(slot, n, dev), pos, cu, length, B, n, Hq, rope.struct(ps.d, dev), qo, _stream()),
           "kv_pages_write_rope")
    return out


def kv_pages_fork(pages: Pages, parent, child, length, table, pool, pool_n, keep=None, out=None):
    """Requests child [n] begin with the first keep [n] (None: all) tokens of requests parent [n] and share their full pages: length
    [B], table [B,max_pages] (the children's rows are written), pool [n_pages], pool_n [1].  Returns (length after, pool_n after,
    status [n]), all int32; out may name `length` and `pool_n` themselves for the first two."""
    dev = _here()
    ps = pages.struct(dev)
    n, (B, max_pages) = parent.numel(), table.shape
    if out is None:
        out = tuple(torch.empty(m, dtype=torch.int32, device=table.device) for m in (B, 1, n))
    after, free, status = out
    _check(lib().kv_pages_fork(ps, _ints(parent, n, dev), _ints(child, n, dev), None if keep is None else _ints(keep, n, dev), n,
                               _ints(length, B, dev), _ints(table, B * max_pages, dev), B, max_pages, _ints(pool, ps.n_pages, dev),
                               _ints(pool_n, 1, dev), _ints(after, B, dev), _ints(free, 1, dev), _ints(status, n, dev), _stream()),
           "kv_pages_fork")
    return out


def kv_pages_free(keep, length, table, pool, pool_n, P: int, out=None, ws=None):
    """Requests keep their first keep [B] tokens; pages that no table names any more go to the pool [n_pages] (updated in place):
    length [B], table [B,max_pages], pool_n [1], all int32.  Returns (length after, pool_n after, status [B]); out may name `length` and
    `pool_n` themselves for the first two.  ws: workspace of workspace_bytes(OP_PAGES, B, max_pages, n_pages, P); calls that may be in
    flight at the same time need one each."""
    (B, max_pages), n_pages, dev = table.shape, pool.numel(), _here()
    ws = _workspace(ws, workspace_bytes(OP_PAGES, B, max_pages, n_pages, P), table.device)
    if out is None:
        out = tuple(torch.empty(m, dtype=torch.int32, device=table.device) for m in (B, 1, B))
    after, free, status = out
    _check(lib().kv_pages_free(_ints(keep, B, dev), _ints(length, B, dev), _ints(table, B * max_pages, dev), B, max_pages,
                               _ints(pool, n_pages, dev), _ints(pool_n, 1, dev), n_pages, P, _ints(after, B, dev), _ints(free, 1, dev),
                               _ints(status, B, dev), ws.data_ptr(), ws.numel() * ws.element_size(), _stream()), "kv_pages_free")
    return out


def kv_pages_compact(pages: Pages, keep, length, table, pool, pool_n, out=None, ws=None):
    """The tokens with keep [B, max_pages * P] (uint8 or bool) other than zero move together: length [B], table [B,max_pages], pool
    [n_pages], pool_n [1], all int32.  Returns (length, table, pool, pool_n after, status [B]); out may name the inputs themselves for the
    first four.  ws as for kv_pages_free."""
    dev = _here()
    ps = pages.struct(dev)
    B, max_pages = table.shape
    if keep.dtype not in (torch.uint8, torch.bool) or keep.shape != (B, max_pages * ps.P) or keep.get_device() != dev or not keep.is_contiguous():
        raise ValueError(f"keep must be [{B}, {max_pages * ps.P}] bytes, contiguous on the current device")
    ws = _workspace(ws, workspace_bytes(OP_PAGES, B, max_pages, ps.n_pages, ps.P), table.device)
    if out is None:
        i = lambda *n: torch.empty(n, dtype=torch.int32, device=table.device)
        out = (i(B), i(B, max_pages), i(ps.n_pages), i(1), i(B))
    after, table_out, pool_out, free, status = out
    _check(lib().kv_pages_compact(ps, keep.data_ptr(), _ints(length, B, dev), _ints(table, B * max_pages, dev), B, max_pages,
                                  _ints(pool, ps.n_pages, dev), _ints(pool_n, 1, dev), _ints(after, B, dev),
                                  _ints(table_out, B * max_pages, dev), _ints(pool_out, ps.n_pages, dev), _ints(free, 1, dev),
                                  _ints(status, B, dev), ws.data_ptr(), ws.numel() * ws.element_size(), _stream()), "kv_pages_compact")
    return out


def probe_mfma_bf16(iters: int = 20000, random_operands: bool = False) -> float:
    """Measured register-resident bf16 matrix-core rate in TFLOP/s (times one probe launch with events); with
    random_operands the multipliers see data like real keys and queries and the chip holds a lower clock."""
    sink = torch.zeros(1, dtype=torch.float32, device="cuda")
    flops = ctypes.c_double(0.0)
    ro = 1 if random_operands else 0
    _check(lib().fastar_probe_mfma_bf16(200, ro, sink.data_ptr(), ctypes.byref(flops), _stream()), "fastar_probe_mfma_bf16")
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    _check(lib().fastar_probe_mfma_bf16(iters, ro, sink.data_ptr(), ctypes.byref(flops), _stream()), "fastar_probe_mfma_bf16")
    e1.record()
    torch.cuda.synchronize()
    return flops.value / (e0.elapsed_time(e1) * 1e-3) / 1e12


def debug_plan_wait(spin_limit: int = -1, extra_arrivals: int = 0) -> None:
    """Test hook (fastar_debug_plan_wait): bound the eviction plan's waits and add arrivals that never come."""
    _check(lib().fastar_debug_plan_wait(spin_limit, extra_arrivals), "fastar_debug_plan_wait")


ATTN_KERNELS = ("plain", "waves", "one", "one_shared", "pair", "pair_split")   # as fastar_probe_attn_route numbers them


def attn_route(n_items: int, d: int, BQ: int, BK: int, n_sel: int, ws: bool) -> tuple[str, int]:
    """Which kernel a bf16 sparse_attn_fwd call takes for n_items (head, query block) pairs, and its number of wavefronts per
    group, whole blocks per XCD or workgroups per block (fastar_probe.h).  Needs no GPU."""
    n = ctypes.c_int()
    rc = lib().fastar_probe_attn_route(n_items, d, BQ, BK, n_sel, int(ws), ctypes.byref(n))
    if rc < 0:
        _check(rc, "fastar_probe_attn_route")
    return ATTN_KERNELS[rc], n.value


def probe_copy(mib: int = 1024, reps: int = 5) -> float:
    """Measured streaming-copy rate in GB/s (read + write bytes over time)."""
    src = torch.ones(mib << 20, dtype=torch.uint8, device="cuda")
    dst = torch.empty_like(src)
    _check(lib().fastar_probe_copy(src.data_ptr(), dst.data_ptr(), src.numel(), _stream()), "fastar_probe_copy")
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(reps):
        _check(lib().fastar_probe_copy(src.data_ptr(), dst.data_ptr(), src.numel(), _stream()), "fastar_probe_copy")
    e1.record()
    torch.cuda.synchronize()
    return 2.0 * src.numel() * reps / (e0.elapsed_time(e1) * 1e-3) / 1e9
