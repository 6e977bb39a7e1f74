"""Binding of libzipcache.so: argument marshalling only.

Every function has the name of the C entry point it calls.  Tensors are torch
tensors on the GPU (torch supplies device memory and the current HIP stream);
no arithmetic of the method happens here.  The calls of a prompt and of a decode
step are marshalled by native code (`csrc/host/marshal.cpp` -> `_zc_host.so`), the
comparison helpers by ctypes.  If the libraries have not been built the import of
any entry point fails loudly - there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libzipcache.so")
HOST_PATH = os.path.join(_HERE, "_zc_host.so")

ZC_OK = 0
ZC_F32, ZC_F16, ZC_BF16 = 0, 1, 2
ZC_SCHEME_CHANNEL, ZC_SCHEME_CST, ZC_SCHEME_TOKEN = 0, 1, 2
ZC_LAYOUT_ROW, ZC_LAYOUT_TGROUP = 0, 1
ZC_SLOT_ALIGN = 64

SCHEMES = {"channel": ZC_SCHEME_CHANNEL, "cst": ZC_SCHEME_CST, "token": ZC_SCHEME_TOKEN}
_DTYPE = {torch.float32: ZC_F32, torch.float16: ZC_F16, torch.bfloat16: ZC_BF16}


class zc_tensor4(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("dtype", C.c_int32), ("reserved", C.c_int32),
                ("B", C.c_int64), ("H", C.c_int64), ("L", C.c_int64), ("D", C.c_int64),
                ("sB", C.c_int64), ("sH", C.c_int64), ("sL", C.c_int64)]


class zc_packed(C.Structure):
    _fields_ = [("layout", C.c_int32), ("scheme", C.c_int32), ("bits_hi", C.c_int32), ("bits_lo", C.c_int32),
                ("B", C.c_int64), ("H", C.c_int64), ("D", C.c_int64),
                ("cap_hi", C.c_int64), ("cap_lo", C.c_int64), ("n_hi", C.c_int64), ("n_lo", C.c_int64),
                ("codes_hi", C.c_void_p), ("codes_lo", C.c_void_p),
                ("tok_scale_hi", C.c_void_p), ("tok_zero_hi", C.c_void_p),
                ("tok_scale_lo", C.c_void_p), ("tok_zero_lo", C.c_void_p),
                ("pos_hi", C.c_void_p), ("pos_lo", C.c_void_p),
                ("chan_scale", C.c_void_p), ("chan_zero", C.c_void_p),
                ("chunk_table", C.c_void_p), ("chunk_table_host", C.c_void_p),
                ("n_chunks", C.c_int32), ("max_chunks", C.c_int32)]


class ZipCacheError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        msg = load().zc_status_string(status).decode()
        super().__init__(f"{fn} failed with status {status}: {msg}")


_lib = None
_host = None


def load() -> C.CDLL:
    """Loads the HIP library; raises if it has not been built."""
    global _lib, _host
    if _lib is not None:
        return _lib
    for path in (LIB_PATH, HOST_PATH):
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: run `python __graft_entry__.py` to build the HIP library")
    lib = C.CDLL(LIB_PATH)
    P, I32, I64, F, SZ = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
    T4, PK = C.POINTER(zc_tensor4), C.POINTER(zc_packed)
    lib.zc_probe_saliency_workspace.restype = SZ
    lib.zc_probe_saliency_workspace.argtypes = [I64, I64, I64, I64]
    lib.zc_probe_saliency.restype = C.c_int
    lib.zc_probe_saliency.argtypes = [T4, T4, P, P, I32, F, P, P, P, P, SZ, P]
    lib.zc_probe_accumulated.restype = C.c_int
    lib.zc_probe_accumulated.argtypes = [T4, T4, P, P, I32, F, P, P, P, P, SZ, P]
    lib.zc_prefill_attention.restype = C.c_int
    lib.zc_prefill_attention.argtypes = [T4, T4, T4, F, T4, P, P, I32, P, P]
    lib.zc_select_salient_workspace.restype = SZ
    lib.zc_select_salient_workspace.argtypes = [I64, I64]
    lib.zc_select_salient.restype = C.c_int
    lib.zc_select_salient.argtypes = [P, I64, I64, I64, P, P, P, P, SZ, P]
    lib.zc_quantize_pack_workspace.restype = SZ
    lib.zc_quantize_pack_workspace.argtypes = [I64, I64, I64, I64]
    lib.zc_quantize_pack.restype = C.c_int
    lib.zc_quantize_pack.argtypes = [T4, P, I64, P, I64, I64, PK, P, SZ, P]
    lib.zc_quantize_pack_kv_workspace.restype = SZ
    lib.zc_quantize_pack_kv_workspace.argtypes = [I64, I64, I64, I64]
    lib.zc_quantize_pack_kv.restype = C.c_int
    lib.zc_quantize_pack_kv.argtypes = [T4, T4, P, I64, P, I64, I64, PK, PK, P, SZ, P]
    lib.zc_decode_attention_workspace.restype = SZ
    lib.zc_decode_attention_workspace.argtypes = [I64, I64, I64]
    lib.zc_decode_attention.restype = C.c_int
    lib.zc_decode_attention.argtypes = [T4, PK, PK, T4, T4, I64, F, P, P, P, SZ, P]
    lib.zc_decode_attention_static.restype = C.c_int
    lib.zc_decode_attention_static.argtypes = [T4, PK, PK, T4, T4, I64, F, P, P, P]
    lib.zc_decode_probs.restype = C.c_int
    lib.zc_decode_probs.argtypes = [T4, PK, T4, I64, I64, F, P, P, I64, P]
    lib.zc_rows_saliency.restype = C.c_int
    lib.zc_rows_saliency.argtypes = [P, P, I32, I64, I64, I64, I64, I32, P, P]
    lib.zc_dequantize_cache.restype = C.c_int
    lib.zc_dequantize_cache.argtypes = [PK, T4, P]
    lib.zc_group_quantize.restype = C.c_int
    lib.zc_group_quantize.argtypes = [T4, P, I64, I32, I32, P, P, P, P, P]
    lib.zc_unpack.restype = C.c_int
    lib.zc_unpack.argtypes = [PK, I32, I32, P, P, P]
    lib.zc_paged_tables.restype = C.c_int
    lib.zc_paged_tables.argtypes = [P, P, I64, P, I64, I64, P, I64, P, I64, P, P, I64, P, P]
    lib.zc_paged_store.restype = C.c_int
    lib.zc_paged_store.argtypes = [T4, T4, P, T4, T4, P]
    lib.zc_paged_load.restype = C.c_int
    lib.zc_paged_load.argtypes = [T4, T4, P, I64, I64, P, T4, T4, P]
    lib.zc_paged_attention_workspace.restype = SZ
    lib.zc_paged_attention_workspace.argtypes = [I64, I64, I64, I64, I64]
    lib.zc_paged_attention.restype = C.c_int
    lib.zc_paged_attention.argtypes = [T4, T4, T4, P, I64, I64, P, P, I64, I32, I32, F, T4, P, P, SZ, P]
    lib.zc_paged_shared_attention_workspace.restype = SZ
    lib.zc_paged_shared_attention_workspace.argtypes = [I64, I64, I64, I64, I64, I64]
    lib.zc_paged_shared_attention.restype = C.c_int
    lib.zc_paged_shared_attention.argtypes = [T4, T4, T4, P, I64, I64, P, P, I64, P, I64, I64, P, P, I64, F, T4, P, P, SZ, P]
    lib.zc_paged_scores.restype = C.c_int
    lib.zc_paged_scores.argtypes = [T4, T4, P, I64, I64, P, P, I64, I32, I32, F, P, F, P, P]
    lib.zc_paged_evict_workspace.restype = SZ
    lib.zc_paged_evict_workspace.argtypes = [I64, I64, I64, I64, I32]
    lib.zc_paged_evict.restype = C.c_int
    lib.zc_paged_evict.argtypes = [T4, T4, P, P, I64, I64, P, P, I64, I64, I32, I32, I32, P, P, P, I64, P, P, P, SZ, P]
    lib.zc_arena_bytes.restype = SZ
    lib.zc_arena_bytes.argtypes = [I64, I64, I64, I64, I32]
    lib.zc_arena_slots.restype = I64
    lib.zc_arena_slots.argtypes = [I64, I64]
    lib.zc_status_string.restype = C.c_char_p
    lib.zc_status_string.argtypes = [C.c_int]
    lib.zc_version.restype = C.c_int
    lib.zc_version.argtypes = []
    if _host is None:
        spec = importlib.util.spec_from_file_location("paper_2405_14256_amd._zc_host", HOST_PATH)
        host = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(host)
    else:
        host = _host
    host.bind(tuple(C.cast(getattr(lib, name), C.c_void_p).value for name in host.names()))
    _lib, _host = lib, host
    return lib


def _native():
    """The native marshalling module, bound to the loaded library."""
    if _lib is None:
        load()
    return _host


def _check(fn: str, status: int) -> None:
    if status != ZC_OK:
        raise ZipCacheError(fn, status)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def tensor4(t: torch.Tensor) -> zc_tensor4:
    """Describes a [B, H, L, D] torch tensor (any strides, unit stride on D)."""
    assert t.dim() == 4 and t.stride(3) == 1, "need a 4-D tensor with contiguous last axis"
    return zc_tensor4(t.data_ptr(), _DTYPE[t.dtype], 0, t.shape[0], t.shape[1], t.shape[2], t.shape[3],
                      t.stride(0), t.stride(1), t.stride(2))


class PackedTensor:
    """Caller-side owner of the arrays of one zc_packed (K or V of a cache)."""

    def __init__(self, B: int, H: int, D: int, cap_hi: int, cap_lo: int, bits_hi: int, bits_lo: int,
                 scheme: str, layout: int, max_chunks: int = 8, device="cuda", store_pos: bool = True):
        lib = load()
        self.B, self.H, self.D = B, H, D
        al = ZC_SLOT_ALIGN
        cap_hi = (cap_hi + al - 1) // al * al
        cap_lo = (cap_lo + al - 1) // al * al
        dev = torch.device(device)
        W = H * D
        self.codes_hi = torch.zeros(max(lib.zc_arena_bytes(B, H, D, cap_hi, bits_hi), 16), dtype=torch.uint8, device=dev)
        self.codes_lo = torch.zeros(max(lib.zc_arena_bytes(B, H, D, cap_lo, bits_lo), 16), dtype=torch.uint8, device=dev)
        f32 = dict(dtype=torch.float32, device=dev)
        self.tok_scale_hi = torch.zeros(B, max(cap_hi, 1), **f32)
        self.tok_zero_hi = torch.zeros(B, max(cap_hi, 1), **f32)
        self.tok_scale_lo = torch.zeros(B, max(cap_lo, 1), **f32)
        self.tok_zero_lo = torch.zeros(B, max(cap_lo, 1), **f32)
        self.pos_hi = torch.full((B, max(cap_hi, 1)), -1, dtype=torch.int32, device=dev) if store_pos else None
        self.pos_lo = torch.full((B, max(cap_lo, 1)), -1, dtype=torch.int32, device=dev) if store_pos else None
        self.chan_scale = torch.zeros(max_chunks, 2, B, W, **f32)
        self.chan_zero = torch.zeros(max_chunks, 2, B, W, **f32)
        self.chunk_table = torch.zeros(max_chunks, 4, dtype=torch.int32, device=dev)
        self.chunk_table_host = np.zeros((max_chunks, 4), np.int32)
        self.c = zc_packed(layout, SCHEMES[scheme], bits_hi, bits_lo, B, H, D, cap_hi, cap_lo, 0, 0,
                           _ptr(self.codes_hi), _ptr(self.codes_lo),
                           _ptr(self.tok_scale_hi), _ptr(self.tok_zero_hi),
                           _ptr(self.tok_scale_lo), _ptr(self.tok_zero_lo),
                           _ptr(self.pos_hi), _ptr(self.pos_lo),
                           _ptr(self.chan_scale), _ptr(self.chan_zero),
                           _ptr(self.chunk_table), self.chunk_table_host.ctypes.data, 0, max_chunks)
        self.scheme, self.layout = scheme, layout

    def reset(self) -> None:
        """Forget all chunks (the arrays are reused)."""
        self.c.n_hi = self.c.n_lo = 0
        self.c.n_chunks = 0

    def clone(self) -> "PackedTensor":
        """A copy with arrays of its own (same contents, same chunks)."""
        o = PackedTensor(self.B, self.H, self.D, self.c.cap_hi, self.c.cap_lo, self.c.bits_hi, self.c.bits_lo,
                         self.scheme, self.layout, max_chunks=self.c.max_chunks, device=self.chan_scale.device,
                         store_pos=self.pos_hi is not None)
        for name in ("codes_hi", "codes_lo", "tok_scale_hi", "tok_zero_hi", "tok_scale_lo", "tok_zero_lo",
                     "pos_hi", "pos_lo", "chan_scale", "chan_zero", "chunk_table"):
            src = getattr(self, name)
            if src is not None:
                getattr(o, name).copy_(src)
        o.chunk_table_host[:] = self.chunk_table_host
        o.c.n_hi, o.c.n_lo, o.c.n_chunks = self.c.n_hi, self.c.n_lo, self.c.n_chunks
        return o

    @property
    def chunks(self):
        return [tuple(int(v) for v in self.chunk_table_host[i]) for i in range(self.c.n_chunks)]


def zc_probe_saliency(q: torch.Tensor, k: torch.Tensor, probe_pos: torch.Tensor,
                      probe_rows: Optional[torch.Tensor] = None, sm_scale: float = 0.0,
                      lse_ext: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None,
                      scores_per_head: Optional[torch.Tensor] = None, _entry: str = "zc_probe_saliency") -> torch.Tensor:
    host = _native()
    if scores is None:
        scores = torch.empty(q.shape[0], k.shape[2], dtype=torch.float32, device=q.device)
    _check(_entry, host.probe(_entry == "zc_probe_accumulated", q, k, probe_rows, probe_pos, sm_scale, lse_ext, scores, scores_per_head))
    return scores


def zc_probe_accumulated(q: torch.Tensor, k: torch.Tensor, probe_pos: torch.Tensor, **kw) -> torch.Tensor:
    """Eq. 7: as zc_probe_saliency, without the division by the unmasked count."""
    return zc_probe_saliency(q, k, probe_pos, _entry="zc_probe_accumulated", **kw)


def zc_prefill_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, sm_scale: float = 0.0,
                         out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         probe_pos: Optional[torch.Tensor] = None, lse_probe: Optional[torch.Tensor] = None):
    """(out [B, Hq, L, D], lse [B, Hq, L], lse_probe [B, Hq, P] or None)."""
    host = _native()
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    if lse_probe is None and probe_pos is not None and probe_pos.numel():
        lse_probe = torch.empty(q.shape[0], q.shape[1], probe_pos.numel(), dtype=torch.float32, device=q.device)
    _check("zc_prefill_attention", host.prefill(q, k, v, sm_scale, out, lse, probe_pos, lse_probe))
    return out, lse, lse_probe


def zc_select_salient(scores: torch.Tensor, k: int, salient_idx: Optional[torch.Tensor] = None,
                      regular_idx: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None):
    host = _native()
    if salient_idx is None or regular_idx is None:
        B, L = scores.shape
        if salient_idx is None:
            salient_idx = torch.empty(B, max(k, 0), dtype=torch.int32, device=scores.device)
        if regular_idx is None:
            regular_idx = torch.empty(B, max(L - k, 0), dtype=torch.int32, device=scores.device)
    _check("zc_select_salient", host.select(scores, k, salient_idx, regular_idx, mask))
    return salient_idx, regular_idx


def zc_quantize_pack(x: torch.Tensor, salient_idx: torch.Tensor, regular_idx: torch.Tensor,
                     out: PackedTensor, pos_offset: int = 0) -> None:
    _check("zc_quantize_pack", _native().quantize(x, salient_idx, regular_idx, out.c, pos_offset))


def zc_quantize_pack_kv(xk: torch.Tensor, xv: torch.Tensor, salient_idx: torch.Tensor, regular_idx: torch.Tensor,
                        outK: PackedTensor, outV: PackedTensor, pos_offset: int = 0) -> None:
    """Keys and values of one cache in the same launches (the four quantizer calls of Algorithm 2)."""
    _check("zc_quantize_pack_kv", _native().quantize_kv(xk, xv, salient_idx, regular_idx, outK.c, outV.c, pos_offset))


def zc_unpack(p: PackedTensor, which: int, chunk: int, codes: bool = True, dequant: bool = True):
    """(codes uint8 [B, len, W] or None, x_hat float32 [B, len, W] or None) of subset
    `which` (0 hi, 1 lo) of chunk `chunk`, token-major in slot order."""
    lib = load()
    row = p.chunks[chunk]
    n = int(row[2 * which + 1])
    W = p.H * p.D
    dev = p.chan_scale.device
    co = torch.empty(p.B, n, W, dtype=torch.uint8, device=dev) if codes else None
    dq = torch.empty(p.B, n, W, dtype=torch.float32, device=dev) if dequant else None
    _check("zc_unpack", lib.zc_unpack(C.byref(p.c), which, chunk, _ptr(co) if n else None, _ptr(dq) if n else None, _stream()))
    return co, dq


def zc_decode_attention(q: torch.Tensor, Kp: PackedTensor, Vp: PackedTensor,
                        tail_k: Optional[torch.Tensor] = None, tail_v: Optional[torch.Tensor] = None,
                        tail_len: int = 0, sm_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                        lse_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q: [B, Hq, D] or [B, Hq, 1, D]."""
    host = _native()
    if out is None:
        out = torch.empty(q.shape[0], q.shape[1], q.shape[-1], dtype=q.dtype, device=q.device)
    _check("zc_decode_attention", host.decode(False, q, Kp.c, Vp.c, tail_k, tail_v, tail_len, sm_scale, out, lse_out))
    return out


def zc_decode_attention_static(q: torch.Tensor, Kp: PackedTensor, Vp: PackedTensor,
                               tail_k: Optional[torch.Tensor] = None, tail_v: Optional[torch.Tensor] = None,
                               tail_len: int = 0, sm_scale: float = 0.0, *, out: torch.Tensor,
                               lse_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """zc_decode_attention on the library's own scratch buffer: nothing is allocated, here
    or in the library (`out` must be given)."""
    _check("zc_decode_attention_static",
           _native().decode(True, q, Kp.c, Vp.c, tail_k, tail_v, tail_len, sm_scale, out, lse_out))
    return out


def zc_decode_probs(q: torch.Tensor, Kp: PackedTensor, tail_k: Optional[torch.Tensor], tail_len: int, tail_pos0: int,
                    lse: torch.Tensor, probs_out: torch.Tensor, sm_scale: float = 0.0) -> torch.Tensor:
    """probs_out [B, Hq, N] (token order) of one decode step; lse from zc_decode_attention."""
    _check("zc_decode_probs", _native().probs(q, Kp.c, tail_k, tail_len, tail_pos0, lse, probs_out, sm_scale))
    return probs_out


def zc_rows_saliency(rows: torch.Tensor, row_len: torch.Tensor, n_out: int, normalize: bool = True,
                     scores: Optional[torch.Tensor] = None) -> torch.Tensor:
    """rows [P, B, Hq, N] float32, row_len int32 [P] -> scores [B, n_out]."""
    host = _native()
    if scores is None:
        scores = torch.empty(rows.shape[1], n_out, dtype=torch.float32, device=rows.device)
    _check("zc_rows_saliency", host.rows_saliency(rows, row_len, n_out, normalize, scores))
    return scores


def zc_dequantize_cache(p: PackedTensor, out: torch.Tensor) -> torch.Tensor:
    """Scatters x_hat of every token of `p` to out[b, h, position, :]."""
    _check("zc_dequantize_cache", _native().dequantize(p.c, out))
    return out


def zc_group_quantize(x: torch.Tensor, bits: int, group: int = 32, idx: Optional[torch.Tensor] = None,
                      codes: bool = True, dequant: bool = True):
    """Groupwise quantization of the token rows `idx` [B, n] (default: all) of x [B, H, L, D]:
    (codes uint8 [B, n, W], scale [B, n, W/group], zero, x_hat float32 [B, n, W])."""
    lib = load()
    B, H, L, D = x.shape
    n = int(idx.shape[1]) if idx is not None else L
    W = H * D
    dev = x.device
    co = torch.empty(B, n, W, dtype=torch.uint8, device=dev) if codes else None
    sc = torch.empty(B, n, W // group, dtype=torch.float32, device=dev)
    ze = torch.empty(B, n, W // group, dtype=torch.float32, device=dev)
    dq = torch.empty(B, n, W, dtype=torch.float32, device=dev) if dequant else None
    tx = tensor4(x)
    _check("zc_group_quantize", lib.zc_group_quantize(C.byref(tx), _ptr(idx), n, bits, group, _ptr(co), _ptr(sc), _ptr(ze),
                                                      _ptr(dq), _stream()))
    return co, sc, ze, dq


def zc_paged_tables(q_len: torch.Tensor, kv_len: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor, page: int, T: int,
                    n_free: Optional[torch.Tensor] = None, q_start: Optional[torch.Tensor] = None,
                    slot_map: Optional[torch.Tensor] = None, n_taken: Optional[torch.Tensor] = None):
    """One step's bookkeeping from the requests' lengths (int32 [R] each): new pages go into block_table [R, max_blocks];
    returns (q_start [R + 1], slot_map [T], n_taken [1])."""
    status, q_start, slot_map, n_taken = _native().paged_tables(q_len, kv_len, block_table, free_pages, n_free, page, T, q_start, slot_map, n_taken)
    _check("zc_paged_tables", status)
    return q_start, slot_map, n_taken


def zc_paged_store(k: torch.Tensor, v: torch.Tensor, slot_map: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor) -> None:
    """New tokens' k, v [T, Hkv, D] (or [1, Hkv, T, D]) to their slots of the pools [N, Hkv, page, D]."""
    _check("zc_paged_store", _native().paged_store(k, v, slot_map, k_pages, v_pages))


def zc_paged_load(k_pages: torch.Tensor, v_pages: torch.Tensor, block_table: torch.Tensor, kv_len: torch.Tensor, L: Optional[int] = None,
                  k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """(k, v) [R, Hkv, L, D]: the tokens of every request; rows past kv_len are not written."""
    host = _native()
    if k_out is None or v_out is None:
        if L is None:
            given = k_out if k_out is not None else v_out
            L = block_table.shape[1] * k_pages.shape[2] if given is None else given.shape[2]
        shape = (block_table.shape[0], k_pages.shape[1], L, k_pages.shape[3])
        k_out = torch.empty(shape, dtype=k_pages.dtype, device=k_pages.device) if k_out is None else k_out
        v_out = torch.empty(shape, dtype=v_pages.dtype, device=v_pages.device) if v_out is None else v_out
    _check("zc_paged_load", host.paged_load(k_pages, v_pages, block_table, kv_len, k_out, v_out))
    return k_out, v_out


def zc_paged_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, block_table: torch.Tensor, q_start: torch.Tensor,
                       kv_len: torch.Tensor, window: int = 0, sinks: int = 0, sm_scale: float = 0.0,
                       out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
    """q [T, Hq, D] (or [1, Hq, T, D]): a step's new tokens, request after request -> (out like q, lse [Hq, T]).
    Rows behind the last request are not written.  The launch is chosen by the table's room, not by kv_len: pass the
    columns that the longest request needs (block_table[:, :n]) where that is known."""
    host = _native()
    if out is None:
        out = torch.empty_like(q)
    if lse is None and q.dim() in (3, 4):
        T, Hq = (q.shape[0], q.shape[1]) if q.dim() == 3 else (q.shape[2], q.shape[1])
        lse = torch.empty(Hq, T, dtype=torch.float32, device=q.device)
    _check("zc_paged_attention", host.paged_attention(q, k_pages, v_pages, block_table, q_start, kv_len, window, sinks, sm_scale, out, lse))
    return out, lse


def zc_paged_shared_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, prefix_table: torch.Tensor, prefix_len: torch.Tensor,
                              group_start: torch.Tensor, block_table: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor,
                              sm_scale: float = 0.0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
    """zc_paged_attention where requests group_start[g] .. group_start[g + 1] - 1 see, in front of their own kv_len tokens, the prefix_len[g]
    tokens in the pages of prefix_table[g]: these are read and multiplied once for all of the group's rows -> (out like q, lse [Hq, T])."""
    host = _native()
    if out is None:
        out = torch.empty_like(q)
    if lse is None and q.dim() in (3, 4):
        T, Hq = (q.shape[0], q.shape[1]) if q.dim() == 3 else (q.shape[2], q.shape[1])
        lse = torch.empty(Hq, T, dtype=torch.float32, device=q.device)
    _check("zc_paged_shared_attention", host.paged_shared(q, k_pages, v_pages, prefix_table, prefix_len, group_start, block_table, q_start, kv_len,
                                                          sm_scale, out, lse))
    return out, lse


def zc_paged_scores(q: torch.Tensor, k_pages: torch.Tensor, block_table: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor,
                    lse: torch.Tensor, scores: torch.Tensor, window: int = 0, sinks: int = 0, sm_scale: float = 0.0,
                    decay: float = 1.0) -> torch.Tensor:
    """Adds a step's attention weights to the scores [N, Hkv, page] of the tokens they went to; q, lse [Hq, T] as in zc_paged_attention.
    A step's new tokens start from 0 (whatever their places held), the others from decay times what they had."""
    _check("zc_paged_scores", _native().paged_scores(q, k_pages, block_table, q_start, kv_len, lse, scores, window, sinks, sm_scale, decay))
    return scores


def zc_paged_evict(k_pages: torch.Tensor, v_pages: torch.Tensor, scores: torch.Tensor, block_table: torch.Tensor, kv_len: torch.Tensor,
                   keep: torch.Tensor, most: int, sinks: int = 0, recent: int = 0, together: bool = False,
                   free_pages: Optional[torch.Tensor] = None, n_free: Optional[torch.Tensor] = None, new_len: Optional[torch.Tensor] = None,
                   kept: Optional[torch.Tensor] = None, n_freed: Optional[torch.Tensor] = None):
    """Of request r's kv_len[r] tokens keep[r] at most (and `most`, which the host knows) stay, by scores [N, Hkv, page]; keys, values and
    scores move to the front of its pages.  Returns (new_len [R], kept [R, Hkv, most] - [R, 1, most] with `together` - and n_freed [1],
    None without a list of free pages)."""
    host = _native()
    R, dev = block_table.shape[0], k_pages.device
    if new_len is None:
        new_len = torch.empty(R, dtype=torch.int32, device=dev)
    if kept is None:
        kept = torch.empty(R, 1 if together else k_pages.shape[1], max(most, 0), dtype=torch.int32, device=dev)
    if n_freed is None and free_pages is not None:
        n_freed = torch.empty(1, dtype=torch.int32, device=dev)
    _check("zc_paged_evict", host.paged_evict(k_pages, v_pages, scores, block_table, kv_len, keep, most, sinks, recent, together, new_len, kept,
                                              free_pages, n_free, n_freed))
    return new_len, kept, n_freed
