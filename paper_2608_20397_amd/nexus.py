"""ctypes binding of libnexus (include/nexus.h): argument marshalling only.

Every step of the path runs in the library's HIP kernels.  torch provides device memory and the
current stream; this module builds the C descriptors from tensors, calls the C entry points on
``torch.cuda.current_stream()`` and turns a non-zero status into :class:`NexusError`.  If the
shared library has not been built, :func:`lib` raises: there is no fallback.
"""

from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass, field

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnexus.so")

OK, EINVAL, ESHAPE, EDTYPE, EROPE, ERANGE, ELAYOUT, EWORKSPACE, EHIP = range(9)
BF16, F32 = 0, 1
V_ROWMAJOR, V_TRANSPOSED = 0, 1
ROPE_NEOX, ROPE_INTERLEAVED = 0, 1
PAGE = 16


class NexusError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        msg = lib().nexus_status_str(status).decode()
        super().__init__(f"{what}: status {status} ({msg})" if what else f"status {status} ({msg})")


class CBlock(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_layers", C.c_int32),
                ("n_tokens", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("rope_style", C.c_int32), ("base_pos", C.c_int64),
                ("rope_base", C.c_double)]


class CKvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_layers", C.c_int32),
                ("n_phys_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("v_layout", C.c_int32),
                ("rope_style", C.c_int32), ("rope_base", C.c_double)]


class CKv8Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("n_layers", C.c_int32), ("n_phys_pages", C.c_int32),
                ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("rope_style", C.c_int32), ("rope_base", C.c_double)]


class CPageTable(C.Structure):
    _fields_ = [("map", C.c_void_p), ("n_logical_pages", C.c_int32)]


_lib = None


def lib():
    """Load libnexus.so (built by ``paper_2608_20397_amd.build``); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2608_20397_amd.build`")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, f32, f64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_double, C.c_size_t
    pB, pC, pT = C.POINTER(CBlock), C.POINTER(CKvCache), C.POINTER(CPageTable)
    p8, pI32, pI64 = C.POINTER(CKv8Cache), C.POINTER(C.c_int32), C.POINTER(C.c_int64)
    sigs = {
        "nexus_abi_version": (i32, []),
        "nexus_status_str": (C.c_char_p, [i32]),
        "nexus_redecode_len": (i64, [i64, i64, i32, i32, i32]),
        "nexus_check_page_table": (i32, [C.POINTER(C.c_int32), i32, i32]),
        "nexus_rephase_k": (i32, [pB, i64, i64, f64, vp]),
        "nexus_rephase_k_paged": (i32, [pC, pT, i64, i32, i64, i64, f64, vp]),
        "nexus_splice_pages": (i32, [pC, pT, pB, i64, vp]),
        "nexus_splice_rephase_pages": (i32, [pC, pT, pB, i64, i64, vp]),
        "nexus_rope_append": (i32, [pC, pT, vp, vp, i32, i64, i64, vp]),
        "nexus_suffix_attn": (i32, [vp, i32, i32, pC, pT, i32, i64, f32, i32, f32, vp, vp, sz, vp]),
        "nexus_suffix_attn_workspace": (sz, [i32, i32, pC, i64]),
        "nexus_suffix_attn_noalloc": (i32, [vp, i32, i32, pC, pT, i32, i64, f32, i32, f32, vp,
                                            vp]),
        "nexus_suffix_attn_varlen": (i32, [vp, i32, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                           C.POINTER(C.c_int64), i32, pC, pT, i32, f32, i32, f32,
                                           vp, vp, sz, vp]),
        "nexus_suffix_attn_varlen_workspace": (sz, [i32, C.POINTER(C.c_int32),
                                                    C.POINTER(C.c_int32), C.POINTER(C.c_int64),
                                                    i32, pC]),
        "nexus_decode_attn": (i32, [vp, i32, i32, pC, vp, i32, vp, i32, i32, f32, i32, f32, vp,
                                    vp, sz, vp]),
        "nexus_decode_attn_workspace": (sz, [i32, i32, pC, i32]),
        "nexus_kv8_append": (i32, [p8, pT, vp, vp, i32, i32, i64, i64, vp]),
        "nexus_kv8_append_step": (i32, [p8, vp, i32, vp, i32, i32, vp, vp, i32, vp]),
        "nexus_kv8_splice": (i32, [p8, pT, pB, i64, i64, vp]),
        "nexus_kv8_read": (i32, [p8, pT, i64, i32, i32, vp, vp, vp]),
        "nexus_kv8_suffix_attn": (i32, [vp, i32, i32, p8, pT, i32, i64, f32, f32, vp, vp, sz, vp]),
        "nexus_kv8_suffix_attn_workspace": (sz, [i32, i32, p8, i64]),
        "nexus_kv8_suffix_attn_varlen": (i32, [vp, i32, pI32, pI32, pI64, i32, p8, pT, i32, f32,
                                               f32, vp, vp, sz, vp]),
        "nexus_kv8_suffix_attn_varlen_workspace": (sz, [i32, pI32, pI32, pI64, i32, p8]),
        "nexus_kv8_decode_attn": (i32, [vp, i32, i32, p8, vp, i32, vp, i32, i32, f32, f32, vp, vp,
                                        sz, vp]),
        "nexus_kv8_decode_attn_workspace": (sz, [i32, i32, p8, i32]),
        "nexus_batch_pages": (i32, [vp, vp, i32, vp, vp, i32, vp, i32, i32, vp, vp, vp, vp, vp, vp]),
        # (the calls of a round take the cache's descriptor as packed bytes)
        "nexus_norm_rope_append": (i32, [vp, i32, vp, i64, vp, i64, vp, i64, i32, i32, vp, vp, f32, vp, vp,
                                         vp, vp]),
        "nexus_window_attn": (i32, [vp, i32, i32, vp, vp, i32, vp, vp, i32, i32, i32, i32, i32, f32, i32, f32,
                                    vp, vp, sz, vp]),
        "nexus_window_attn_workspace": (sz, [i32, i32, vp, i32, i32, i32, i32]),
        "nexus_window_decode_attn": (i32, [vp, i32, i32, vp, vp, i32, vp, i32, i32, i32, i32, f32, i32, f32, vp,
                                           vp, sz, vp]),
        "nexus_window_decode_attn_workspace": (sz, [i32, i32, vp, i32, i32, i32]),
        "nexus_kv_copy_tokens": (i32, [pC, vp, vp, i32, i64, i32, vp]),
        "nexus_kv_share_prefix": (i32, [pC, vp, vp, i32, i32, vp]),
        "nexus_l0_longest_prefix": (i32, [C.POINTER(C.c_int32), i32, C.POINTER(C.c_int32),
                                          C.POINTER(C.c_int32), i32, i32,
                                          C.POINTER(C.c_int32), C.POINTER(C.c_int32)]),
        "nexus_slb_quantize": (i32, [vp, i32, i32, vp, vp, vp]),
        "nexus_slb_scan": (i32, [vp, vp, i32, vp, vp, i32, i32, i32, f32, vp, vp, vp, vp, vp, sz,
                                 vp]),
        "nexus_slb_scan_workspace": (sz, [i32, i32, i32, i32]),
        "nexus_calib_copy": (i32, [vp, vp, sz, vp]),
        "nexus_calib_mfma_bf16": (i32, [i32, vp, C.POINTER(C.c_double), vp]),
        "nexus_calib_lds_dma": (i32, [vp, sz, vp]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _check(status: int, what: str):
    if status != OK:
        raise NexusError(status, what)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise NexusError(EDTYPE, f"unsupported dtype {t.dtype}")


# Both return plain integers, which ctypes passes for a void pointer: an object for each of a call's ten
# pointers and a Stream object for its stream took 6 of the 29 us that quantising one query and scanning
# 250 tools cost the host.  The raw stream has no public accessor; without it the Stream object serves.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


# torch.cuda.current_device without its look whether the driver is there (a device tensor says so); no public accessor
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _current_device() -> int:
    return torch.cuda.current_device() if _get_device is None else _get_device()


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


def _ptr(t):
    return t.data_ptr() if t is not None else 0


def _on_device(*named):
    """Every given (name, tensor) pair must be a device tensor, all on one device; returns that
    device.  The kernels dereference every pointer they get as a device address, so a host
    tensor must never reach them."""
    dev = None
    for name, t in named:
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise NexusError(EINVAL, f"{name} must be a device tensor")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise NexusError(EINVAL, f"{name} is on {t.device}, the other operands on {dev}")
    return dev


def _checked_map(cache, k: torch.Tensor, pm: torch.Tensor) -> CPageTable:
    if pm.dtype != torch.int32 or pm.dim() != 1 or not pm.is_contiguous():
        raise NexusError(EINVAL, "page_map must be a contiguous int32 vector")
    _on_device(("cache k", k), ("page_map", pm))
    npp = k.shape[1]
    if pm.is_inference():                            # has no version counter: its changes cannot be noticed
        check_page_table(pm.cpu().numpy(), npp)
        return CPageTable(pm.data_ptr(), pm.numel())
    key = (pm.data_ptr(), pm._version, pm.numel(), npp)
    if cache._map_checked is None or cache._map_checked[0] != key:
        check_page_table(pm.cpu().numpy(), npp)      # raises NexusError(ERANGE)
        cache._map_checked = (key, pm)               # pm is kept, so no other map can get its address
    return CPageTable(pm.data_ptr(), pm.numel())


@dataclass
class Block:
    """A compiled KV block in HBM: k, v [n_layers][n_tokens][n_kv_heads][head_dim]."""
    k: torch.Tensor
    v: torch.Tensor
    base_pos: int
    rope_base: float
    rope_style: int = ROPE_NEOX

    def c(self) -> CBlock:
        L, T, H, D = self.k.shape
        if tuple(self.v.shape) != (L, T, H, D) or not (self.k.is_contiguous() and self.v.is_contiguous()):
            raise NexusError(ESHAPE, "block k/v must be contiguous [L][T][H][D] of equal shape")
        _on_device(("block k", self.k), ("block v", self.v))
        return CBlock(self.k.data_ptr(), self.v.data_ptr(), L, T, H, D, _dtype_code(self.k),
                      self.rope_style, self.base_pos, self.rope_base)


@dataclass
class PagedKVCache:
    """k [L][n_phys_pages][H][16][D]; v the same or, transposed, [L][H][D][n_phys_pages*16];
    page_map int32 [n_logical_pages] on the device.

    The kernels read the page map's entries on the device without a host check, so the map is
    validated here (``nexus_check_page_table`` on a host copy: every entry a distinct physical
    page) the first time a call uses it and again whenever it has changed since (another tensor,
    or an in-place write that bumped its version counter).  A map made under torch.inference_mode keeps
    no such counter and is copied to the host and validated by every call."""
    k: torch.Tensor
    v: torch.Tensor
    page_map: torch.Tensor
    rope_base: float
    v_layout: int = V_ROWMAJOR
    rope_style: int = ROPE_NEOX
    _map_checked: tuple | None = field(default=None, init=False, repr=False, compare=False)

    def c(self) -> CKvCache:
        k, v = self.k, self.v
        shape = L, npp, H, P, D = k.shape
        if P != PAGE or not (k.is_contiguous() and v.is_contiguous()):
            raise NexusError(ESHAPE, "cache k must be contiguous [L][pages][H][16][D]")
        if not _all_here(k, v, self.page_map):
            _on_device(("cache k", k), ("cache v", v), ("page_map", self.page_map))
        want_v = (L, H, D, npp * P) if self.v_layout == V_TRANSPOSED else shape
        if v.shape != want_v:
            raise NexusError(ESHAPE, f"cache v must be {want_v}, got {tuple(v.shape)}")
        if v.dtype != k.dtype:
            raise NexusError(EDTYPE, "cache k and v dtypes differ")
        return CKvCache(k.data_ptr(), v.data_ptr(), L, npp, P, H, D, _dtype_code(k), self.v_layout,
                        self.rope_style, self.rope_base)

    def pt(self) -> CPageTable:
        return _checked_map(self, self.k, self.page_map)

    @property
    def n_layers(self):
        return self.k.shape[0]


def splice_pages(cache: PagedKVCache, block: Block, offset: int):
    cc, pt, cb = cache.c(), cache.pt(), block.c()
    _on_device(("cache k", cache.k), ("block k", block.k))
    _check(lib().nexus_splice_pages(C.byref(cc), C.byref(pt), C.byref(cb), offset, _stream()),
           "nexus_splice_pages")


def splice_rephase_pages(cache: PagedKVCache, block: Block, offset: int, dst_pos: int):
    """Splice ``block`` at ``offset`` with its keys re-anchored from block.base_pos to
    ``dst_pos`` in the same pass (the block itself is left as it is)."""
    cc, pt, cb = cache.c(), cache.pt(), block.c()
    _on_device(("cache k", cache.k), ("block k", block.k))
    _check(lib().nexus_splice_rephase_pages(C.byref(cc), C.byref(pt), C.byref(cb), offset, dst_pos,
                                            _stream()), "nexus_splice_rephase_pages")


def rope_append(cache: PagedKVCache, k: torch.Tensor, v: torch.Tensor, offset: int, pos0: int):
    """Write un-rotated keys ``k`` (rotated here to positions pos0 + j) and values ``v``, both
    [L][T][H][D] of the cache dtype, into logical slots offset .. offset + T - 1."""
    cc, pt = cache.c(), cache.pt()
    L, T, H, D = k.shape
    if tuple(v.shape) != (L, T, H, D) or not (k.is_contiguous() and v.is_contiguous()):
        raise NexusError(ESHAPE, "k/v must be contiguous [L][T][H][D] of equal shape")
    _on_device(("cache k", cache.k), ("k", k), ("v", v))
    if (L, H, D) != (cc.n_layers, cc.n_kv_heads, cc.head_dim) or _dtype_code(k) != cc.dtype \
            or _dtype_code(v) != cc.dtype:
        raise NexusError(ESHAPE, "k/v must match the cache's layers, heads, head_dim and dtype")
    _check(lib().nexus_rope_append(C.byref(cc), C.byref(pt), _ptr(k), _ptr(v), T, offset, pos0,
                                   _stream()), "nexus_rope_append")


def rephase_k(block: Block, src_pos: int, dst_pos: int, rope_base: float):
    cb = block.c()
    _check(lib().nexus_rephase_k(C.byref(cb), src_pos, dst_pos, rope_base, _stream()),
           "nexus_rephase_k")
    block.base_pos = cb.base_pos


def rephase_k_paged(cache: PagedKVCache, offset: int, n_tokens: int, src_pos: int, dst_pos: int,
                    rope_base: float):
    cc, pt = cache.c(), cache.pt()
    _check(lib().nexus_rephase_k_paged(C.byref(cc), C.byref(pt), offset, n_tokens, src_pos,
                                       dst_pos, rope_base, _stream()), "nexus_rephase_k_paged")


def suffix_attn_workspace_bytes(cache: PagedKVCache, n_s: int, n_q_heads: int, n_past: int) -> int:
    cc = cache.c()
    n = lib().nexus_suffix_attn_workspace(n_s, n_q_heads, C.byref(cc), n_past)
    if n == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_suffix_attn_workspace")
    return n


def _workspace(nbytes: int, device, workspace):
    if nbytes == 0:
        return None
    if workspace is not None:
        return workspace
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def suffix_attn(q: torch.Tensor, cache: PagedKVCache, layer: int, n_past: int,
                softcap: float = 0.0, v_layout: int | None = None, scale: float = 0.0,
                out: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """q [n_s][n_q_heads][D] -> out [n_s][n_q_heads][D] (cache dtype)."""
    n_s, hq, _ = q.shape
    if not q.is_contiguous():
        raise NexusError(EINVAL, "q must be contiguous")
    if q.dtype != cache.k.dtype:
        raise NexusError(EDTYPE, "q dtype differs from the cache")
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise NexusError(EINVAL, "out must be contiguous, shaped and typed like q")
    cc, pt = cache.c(), cache.pt()
    _on_device(("cache k", cache.k), ("q", q), ("out", out), ("workspace", workspace))
    ws_bytes = lib().nexus_suffix_attn_workspace(n_s, hq, C.byref(cc), n_past)
    if ws_bytes == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_suffix_attn_workspace")
    ws = _workspace(ws_bytes, q.device, workspace)
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    _check(lib().nexus_suffix_attn(_ptr(q), n_s, hq, C.byref(cc), C.byref(pt), layer, n_past,
                                   softcap, cache.v_layout if v_layout is None else v_layout,
                                   scale, _ptr(out), _ptr(ws), nbytes, _stream()),
           "nexus_suffix_attn")
    return out


def suffix_attn_noalloc(q: torch.Tensor, cache: PagedKVCache, layer: int, n_past: int,
                        softcap: float = 0.0, v_layout: int | None = None, scale: float = 0.0,
                        out: torch.Tensor | None = None):
    """suffix_attn without a workspace: the split partials live in the library's static device
    array (see nexus_suffix_attn_noalloc); with ``out`` given, nothing is allocated."""
    n_s, hq, _ = q.shape
    if not q.is_contiguous():
        raise NexusError(EINVAL, "q must be contiguous")
    if q.dtype != cache.k.dtype:
        raise NexusError(EDTYPE, "q dtype differs from the cache")
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise NexusError(EINVAL, "out must be contiguous, shaped and typed like q")
    cc, pt = cache.c(), cache.pt()
    _on_device(("cache k", cache.k), ("q", q), ("out", out))
    _check(lib().nexus_suffix_attn_noalloc(_ptr(q), n_s, hq, C.byref(cc), C.byref(pt), layer,
                                           n_past, softcap,
                                           cache.v_layout if v_layout is None else v_layout,
                                           scale, _ptr(out), _stream()),
           "nexus_suffix_attn_noalloc")
    return out


def suffix_attn_varlen_workspace_bytes(cache: PagedKVCache, q_start, seq_len, seq_n_past,
                                       n_q_heads: int) -> int:
    n = len(seq_len)
    cc = cache.c()
    nbytes = lib().nexus_suffix_attn_varlen_workspace(n, (C.c_int32 * n)(*q_start),
                                                      (C.c_int32 * n)(*seq_len),
                                                      (C.c_int64 * n)(*seq_n_past), n_q_heads,
                                                      C.byref(cc))
    if nbytes == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_suffix_attn_varlen_workspace")
    return nbytes


def suffix_attn_varlen(q: torch.Tensor, q_start, seq_len, seq_n_past, cache: PagedKVCache,
                       layer: int, softcap: float = 0.0, v_layout: int | None = None,
                       scale: float = 0.0, out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None):
    """Several suffixes in one launch: rows q_start[b] .. + seq_len[b] at positions
    seq_n_past[b] + i."""
    n = len(seq_len)
    qs = (C.c_int32 * n)(*q_start)
    ls = (C.c_int32 * n)(*seq_len)
    ps = (C.c_int64 * n)(*seq_n_past)
    _, hq, _ = q.shape
    if not q.is_contiguous():
        raise NexusError(EINVAL, "q must be contiguous")
    if q.dtype != cache.k.dtype:
        raise NexusError(EDTYPE, "q dtype differs from the cache")
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise NexusError(EINVAL, "out must be contiguous, shaped and typed like q")
    cc, pt = cache.c(), cache.pt()
    _on_device(("cache k", cache.k), ("q", q), ("out", out), ("workspace", workspace))
    ws_bytes = lib().nexus_suffix_attn_varlen_workspace(n, qs, ls, ps, hq, C.byref(cc))
    if ws_bytes == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_suffix_attn_varlen_workspace")
    ws = _workspace(ws_bytes, q.device, workspace)
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    _check(lib().nexus_suffix_attn_varlen(_ptr(q), n, qs, ls, ps, hq, C.byref(cc), C.byref(pt),
                                          layer, softcap,
                                          cache.v_layout if v_layout is None else v_layout,
                                          scale, _ptr(out), _ptr(ws), nbytes, _stream()),
           "nexus_suffix_attn_varlen")
    return out


def decode_attn_workspace_bytes(cache: PagedKVCache, n_seqs: int, n_q_heads: int,
                                max_seq_len: int) -> int:
    cc = cache.c()
    n = lib().nexus_decode_attn_workspace(n_seqs, n_q_heads, C.byref(cc), max_seq_len)
    if n == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_decode_attn_workspace")
    return n


def decode_attn(q: torch.Tensor, cache: PagedKVCache, maps: torch.Tensor, seq_len: torch.Tensor,
                max_seq_len: int, layer: int, softcap: float = 0.0, v_layout: int | None = None,
                scale: float = 0.0, out: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None):
    """One query per sequence: q [n_seqs][n_q_heads][D] -> out (cache dtype).  ``maps`` is a
    device int32 [n_seqs][map_stride] tensor of per-sequence page maps and ``seq_len`` a device
    int32 [n_seqs] tensor (the cache's own page_map is not used)."""
    n, hq, _ = q.shape
    if not q.is_contiguous():
        raise NexusError(EINVAL, "q must be contiguous")
    if q.dtype != cache.k.dtype:
        raise NexusError(EDTYPE, "q dtype differs from the cache")
    if (maps.dtype != torch.int32 or maps.dim() != 2 or maps.shape[0] != n
            or not maps.is_contiguous() or maps.device != q.device):
        raise NexusError(EINVAL, "maps must be a contiguous int32 [n_seqs][stride] device tensor")
    if (seq_len.dtype != torch.int32 or tuple(seq_len.shape) != (n,)
            or not seq_len.is_contiguous() or seq_len.device != q.device):
        raise NexusError(EINVAL, "seq_len must be a contiguous int32 [n_seqs] device tensor")
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise NexusError(EINVAL, "out must be contiguous, shaped and typed like q")
    cc = cache.c()
    _on_device(("cache k", cache.k), ("q", q), ("maps", maps), ("seq_len", seq_len),
               ("out", out), ("workspace", workspace))
    ws_bytes = lib().nexus_decode_attn_workspace(n, hq, C.byref(cc), max_seq_len)
    if ws_bytes == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_decode_attn_workspace")
    ws = _workspace(ws_bytes, q.device, workspace)
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    _check(lib().nexus_decode_attn(_ptr(q), n, hq, C.byref(cc), _ptr(maps), maps.shape[1],
                                   _ptr(seq_len), max_seq_len, layer, softcap,
                                   cache.v_layout if v_layout is None else v_layout, scale,
                                   _ptr(out), _ptr(ws), nbytes, _stream()),
           "nexus_decode_attn")
    return out


@dataclass
class KV8Cache:
    """A paged cache in 8 bits: k, v [L][n_phys_pages][H][16][D] of torch.float8_e4m3fn (or the
    same bytes as uint8), k_scale, v_scale uint8 [L][n_phys_pages][H][16], one scale 2^(byte - 127)
    for each row (token and head); page_map as PagedKVCache, checked the same way.  V is row-major.

    :meth:`empty` allocates one.  Pages are written by kv8_append, kv8_append_step and kv8_splice,
    read back by kv8_read and attended to by kv8_suffix_attn(_varlen) and kv8_decode_attn."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor
    page_map: torch.Tensor
    rope_base: float
    rope_style: int = ROPE_NEOX
    _map_checked: tuple | None = field(default=None, init=False, repr=False, compare=False)

    @classmethod
    def empty(cls, n_layers: int, n_phys_pages: int, n_kv_heads: int, head_dim: int,
              page_map: torch.Tensor, rope_base: float, rope_style: int = ROPE_NEOX):
        """A cache of unwritten pages on page_map's device."""
        rows = (n_layers, n_phys_pages, n_kv_heads, PAGE)
        new = lambda shape, dt: torch.empty(shape, dtype=dt, device=page_map.device)
        return cls(new((*rows, head_dim), torch.float8_e4m3fn), new((*rows, head_dim), torch.float8_e4m3fn),
                   new(rows, torch.uint8), new(rows, torch.uint8), page_map, rope_base, rope_style)

    def c(self) -> CKv8Cache:
        k, v, ks, vs = self.k, self.v, self.k_scale, self.v_scale
        shape = k.shape
        if len(shape) != 5 or shape[3] != PAGE:
            raise NexusError(ESHAPE, "cache k must be [L][pages][H][16][D]")
        if not _all_here(k, v, ks, vs, self.page_map):
            _here(cache_k=k, cache_v=v, k_scale=ks, v_scale=vs, page_map=self.page_map)
        kd, vd = k.dtype, v.dtype
        if (kd != torch.float8_e4m3fn and kd != torch.uint8) or (vd != torch.float8_e4m3fn and vd != torch.uint8):
            raise NexusError(EDTYPE, f"cache k/v: unsupported dtype {kd}, {vd}")
        if ks.dtype != torch.uint8 or vs.dtype != torch.uint8:
            raise NexusError(EDTYPE, f"k_scale/v_scale: unsupported dtype {ks.dtype}, {vs.dtype}")
        if v.shape != shape or not (k.is_contiguous() and v.is_contiguous()):
            raise NexusError(ESHAPE, f"cache k/v must be contiguous [L][pages][H][16][D], got {tuple(shape)}, "
                                     f"{tuple(v.shape)}")
        rows = shape[:4]
        if ks.shape != rows or vs.shape != rows or not (ks.is_contiguous() and vs.is_contiguous()):
            raise NexusError(ESHAPE, f"k_scale/v_scale must be contiguous [L][pages][H][16], got "
                                     f"{tuple(ks.shape)}, {tuple(vs.shape)}")
        L, npp, H, P, D = shape
        return CKv8Cache(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), L, npp, P, H, D,
                         self.rope_style, self.rope_base)

    def pt(self) -> CPageTable:
        return _checked_map(self, self.k, self.page_map)


def _all_here(*tensors) -> bool:
    """Whether the given tensors (None among them) are all on the current device."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            return False
    return dev >= 0 and dev == _current_device()


def _current_of(*tensors) -> int:
    """The current device's index where the given tensors (None among them) are all on it, else -1."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            return -1
    return dev if dev >= 0 and dev == _current_device() else -1


def _stream_of(dev: int):
    """The current stream of the current device, dev."""
    return _stream() if _raw_stream is None else _raw_stream(dev)


def _here(**tensors):
    """The given tensors must be on the current device, to whose stream the launch goes."""
    dev = None
    for name, t in tensors.items():
        if t is None:
            continue
        if dev is None and t.is_cuda:
            dev = torch.cuda.current_device()
        if not t.is_cuda or t.get_device() != dev:
            raise NexusError(EINVAL, f"{name} is on {t.device}, not on the current device")


def _kv8_rows(cc: CKv8Cache, k: torch.Tensor, v: torch.Tensor):
    """Checks rows [L][n][H][D] beside an 8-bit cache; returns n and their dtype's code."""
    shape = k.shape
    if len(shape) != 4 or shape[0] != cc.n_layers or shape[2] != cc.n_kv_heads or shape[3] != cc.head_dim \
            or v.shape != shape or not (k.is_contiguous() and v.is_contiguous()):
        raise NexusError(ESHAPE, "k/v must be contiguous [L][T][H][D] with the cache's L, H and D")
    if v.dtype != k.dtype:
        raise NexusError(EDTYPE, "k and v dtypes differ")
    if not _all_here(k, v):
        _here(k=k, v=v)
    return shape[1], _dtype_code(k)


def kv8_append(cache: KV8Cache, k: torch.Tensor, v: torch.Tensor, offset: int, pos0: int):
    """Quantise un-rotated keys ``k`` (rotated here to positions pos0 + j) and values ``v``, both
    [L][T][H][D] bf16 or fp32, into logical slots offset .. offset + T - 1."""
    cc, pt = cache.c(), cache.pt()
    n, dt = _kv8_rows(cc, k, v)
    _check(lib().nexus_kv8_append(C.byref(cc), C.byref(pt), _ptr(k), _ptr(v), dt, n, offset, pos0,
                                  _stream()), "nexus_kv8_append")


def kv8_append_step(cache: KV8Cache, maps: torch.Tensor, seq_len: torch.Tensor, max_seq_len: int,
                    k: torch.Tensor, v: torch.Tensor):
    """One new token for each sequence, k, v [L][n_seqs][H][D]: rotated to position seq_len[b] - 1
    and written to that slot of map row b (device int32 ``maps`` [n_seqs][stride] and ``seq_len``
    [n_seqs]; lengths outside [1, max_seq_len] write nothing)."""
    cc = cache.c()
    n, dt = _kv8_rows(cc, k, v)
    _kv8_maps(maps, seq_len, n)
    _check(lib().nexus_kv8_append_step(C.byref(cc), _ptr(maps), maps.shape[1], _ptr(seq_len), n,
                                       max_seq_len, _ptr(k), _ptr(v), dt, _stream()),
           "nexus_kv8_append_step")


def kv8_splice(cache: KV8Cache, block: Block, offset: int, dst_pos: int):
    """Splice ``block`` (bf16 or fp32) at ``offset``, its keys re-anchored from block.base_pos to
    ``dst_pos`` and quantised in the same pass (the block itself is left as it is)."""
    cc, pt, cb = cache.c(), cache.pt(), block.c()
    if block.v.dtype != block.k.dtype:
        raise NexusError(EDTYPE, "block k and v dtypes differ")
    _here(block_k=block.k)
    _check(lib().nexus_kv8_splice(C.byref(cc), C.byref(pt), C.byref(cb), offset, dst_pos, _stream()),
           "nexus_kv8_splice")


def kv8_read(cache: KV8Cache, offset: int, n_tokens: int, dtype: torch.dtype = torch.bfloat16,
             out=None):
    """The values of logical tokens offset .. offset + n_tokens - 1 as (k, v), [L][T][H][D] of
    ``dtype`` (bf16 or fp32; both hold them exactly); ``out`` may hold preallocated (k, v)."""
    cc, pt = cache.c(), cache.pt()
    shape = (cc.n_layers, max(0, n_tokens), cc.n_kv_heads, cc.head_dim)
    if out is None:
        out = tuple(torch.empty(shape, dtype=dtype, device=cache.k.device) for _ in range(2))
    k, v = out
    if tuple(k.shape) != shape or k.dtype != dtype:
        raise NexusError(ESHAPE, f"out must be two {shape} tensors of {dtype}")
    n, dt = _kv8_rows(cc, k, v)
    _check(lib().nexus_kv8_read(C.byref(cc), C.byref(pt), offset, n_tokens, dt, _ptr(k), _ptr(v),
                                _stream()), "nexus_kv8_read")
    return k, v


def _kv8_maps(maps: torch.Tensor, seq_len: torch.Tensor, n: int):
    if not _all_here(maps, seq_len):
        _here(maps=maps, seq_len=seq_len)
    if maps.dtype != torch.int32 or maps.dim() != 2 or maps.shape[0] != n or not maps.is_contiguous():
        raise NexusError(EINVAL, "maps must be a contiguous int32 [n_seqs][stride] device tensor")
    if seq_len.dtype != torch.int32 or seq_len.dim() != 1 or seq_len.shape[0] != n or not seq_len.is_contiguous():
        raise NexusError(EINVAL, "seq_len must be a contiguous int32 [n_seqs] device tensor")


def _kv8_query(q: torch.Tensor, cc: CKv8Cache, out, workspace):
    """Checks q [rows][n_q_heads][D] (bf16), out and workspace; returns out."""
    shape = q.shape
    if len(shape) != 3 or shape[2] != cc.head_dim:
        raise NexusError(ESHAPE, "q must be [rows][n_q_heads][D] with the cache's D")
    if not q.is_contiguous():
        raise NexusError(EINVAL, "q must be contiguous")
    if q.dtype != torch.bfloat16:
        raise NexusError(EDTYPE, "q must be bf16 over an 8-bit cache")
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise NexusError(EINVAL, "out must be contiguous, shaped and typed like q")
    if workspace is not None and not workspace.is_contiguous():
        raise NexusError(EINVAL, "workspace must be contiguous")
    if not _all_here(q, out, workspace):
        _here(q=q, out=out, workspace=workspace)
    return out


def _kv8_workspace(nbytes: int, q: torch.Tensor, workspace):
    """(pointer, bytes) of the caller's workspace, or of one allocated here."""
    if nbytes == (1 << 64) - 1:
        return None, 0             # invalid arguments: the call itself reports which check failed
    ws = _workspace(nbytes, q.device, workspace)
    return ws, ws.numel() * ws.element_size() if ws is not None else 0


def kv8_suffix_attn_workspace_bytes(cache: KV8Cache, n_s: int, n_q_heads: int, n_past: int) -> int:
    cc = cache.c()
    n = lib().nexus_kv8_suffix_attn_workspace(n_s, n_q_heads, C.byref(cc), n_past)
    if n == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_kv8_suffix_attn_workspace")
    return n


def kv8_suffix_attn(q: torch.Tensor, cache: KV8Cache, layer: int, n_past: int, softcap: float = 0.0,
                    scale: float = 0.0, out: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None):
    """suffix_attn over an 8-bit cache: q [n_s][n_q_heads][D] bf16 -> out, alike."""
    cc, pt = cache.c(), cache.pt()
    out = _kv8_query(q, cc, out, workspace)
    n_s, hq, _ = q.shape
    need = lib().nexus_kv8_suffix_attn_workspace(n_s, hq, C.byref(cc), n_past)
    ws, nbytes = _kv8_workspace(need, q, workspace)
    _check(lib().nexus_kv8_suffix_attn(_ptr(q), n_s, hq, C.byref(cc), C.byref(pt), layer, n_past,
                                       softcap, scale, _ptr(out), _ptr(ws), nbytes, _stream()),
           "nexus_kv8_suffix_attn")
    return out


def kv8_suffix_attn_varlen(q: torch.Tensor, q_start, seq_len, seq_n_past, cache: KV8Cache,
                           layer: int, softcap: float = 0.0, scale: float = 0.0,
                           out: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """suffix_attn_varlen over an 8-bit cache."""
    n = len(seq_len)
    if len(q_start) != n or len(seq_n_past) != n:
        raise NexusError(EINVAL, "q_start, seq_len and seq_n_past differ in length")
    cc, pt = cache.c(), cache.pt()
    out = _kv8_query(q, cc, out, workspace)
    _, hq, _ = q.shape
    if any(s + m > q.shape[0] for s, m in zip(q_start, seq_len)):
        raise NexusError(ERANGE, "a sequence's rows lie past q")
    qs, ls, ps = (C.c_int32 * n)(*q_start), (C.c_int32 * n)(*seq_len), (C.c_int64 * n)(*seq_n_past)
    need = lib().nexus_kv8_suffix_attn_varlen_workspace(n, qs, ls, ps, hq, C.byref(cc))
    ws, nbytes = _kv8_workspace(need, q, workspace)
    _check(lib().nexus_kv8_suffix_attn_varlen(_ptr(q), n, qs, ls, ps, hq, C.byref(cc), C.byref(pt),
                                              layer, softcap, scale, _ptr(out), _ptr(ws), nbytes,
                                              _stream()), "nexus_kv8_suffix_attn_varlen")
    return out


def kv8_suffix_attn_varlen_workspace_bytes(cache: KV8Cache, q_start, seq_len, seq_n_past,
                                           n_q_heads: int) -> int:
    n = len(seq_len)
    cc = cache.c()
    nbytes = lib().nexus_kv8_suffix_attn_varlen_workspace(n, (C.c_int32 * n)(*q_start),
                                                          (C.c_int32 * n)(*seq_len),
                                                          (C.c_int64 * n)(*seq_n_past), n_q_heads,
                                                          C.byref(cc))
    if nbytes == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_kv8_suffix_attn_varlen_workspace")
    return nbytes


def kv8_decode_attn_workspace_bytes(cache: KV8Cache, n_seqs: int, n_q_heads: int,
                                    max_seq_len: int) -> int:
    cc = cache.c()
    n = lib().nexus_kv8_decode_attn_workspace(n_seqs, n_q_heads, C.byref(cc), max_seq_len)
    if n == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_kv8_decode_attn_workspace")
    return n


def kv8_decode_attn(q: torch.Tensor, cache: KV8Cache, maps: torch.Tensor, seq_len: torch.Tensor,
                    max_seq_len: int, layer: int, softcap: float = 0.0, scale: float = 0.0,
                    out: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """decode_attn over an 8-bit cache: q [n_seqs][n_q_heads][D] bf16 -> out, alike."""
    cc = cache.c()
    out = _kv8_query(q, cc, out, workspace)
    n, hq, _ = q.shape
    _kv8_maps(maps, seq_len, n)
    need = lib().nexus_kv8_decode_attn_workspace(n, hq, C.byref(cc), max_seq_len)
    ws, nbytes = _kv8_workspace(need, q, workspace)
    _check(lib().nexus_kv8_decode_attn(_ptr(q), n, hq, C.byref(cc), _ptr(maps), maps.shape[1],
                                       _ptr(seq_len), max_seq_len, layer, softcap, scale, _ptr(out),
                                       _ptr(ws), nbytes, _stream()), "nexus_kv8_decode_attn")
    return out


def _map_arg(m: torch.Tensor, what: str):
    if m.dtype != torch.int32 or m.dim() != 1 or not m.is_contiguous() or not m.is_cuda:
        raise NexusError(EINVAL, f"{what} must be a contiguous int32 device vector")
    return _ptr(m)


@dataclass
class BatchRows:
    """The layout of a round, device int32 tensors: q_start [n_seqs + 1], seq_len [n_seqs], pos and slot
    [max_tokens], n_left [1] (see nexus_batch_pages)."""
    q_start: torch.Tensor
    seq_len: torch.Tensor
    pos: torch.Tensor
    slot: torch.Tensor
    n_left: torch.Tensor

    @classmethod
    def empty(cls, n_seqs: int, max_tokens: int, device):
        """Unwritten, in one allocation (the "unsafe" split skips autograd's view tracking, which integers have no use
        for)."""
        parts = (n_seqs + 1, n_seqs, max_tokens, max_tokens, 1)
        return cls(*torch.empty(sum(parts), dtype=torch.int32, device=device).unsafe_split_with_sizes(parts))


_I32 = torch.int32
_TOP = (1 << 31) - 1                                 # of an int32 argument: no window, all tokens
_pack_cache = struct.Struct("PPiiiiiiiid").pack      # nexus_kv_cache


def _int32(x: int) -> int:
    """x, or the end of an int32's range that it lies behind: ctypes would bring it round to a number that is allowed."""
    return x if -_TOP <= x <= _TOP else _TOP if x > 0 else -_TOP


def _descriptor(cache: PagedKVCache) -> bytes:
    """The cache as the C calls take it, checked as PagedKVCache.c() does but for the devices, which the caller checks
    with its other operands (1 us of host time a call less)."""
    k, v = cache.k, cache.v
    shape = k.shape
    if len(shape) != 5 or shape[3] != PAGE or not (k.is_contiguous() and v.is_contiguous()):
        raise NexusError(ESHAPE, "cache k must be contiguous [L][pages][H][16][D]")
    L, npp, H, P, D = shape
    if v.shape != ((L, H, D, npp * P) if cache.v_layout == V_TRANSPOSED else shape):
        raise NexusError(ESHAPE, f"cache v does not fit k and its layout, got {tuple(v.shape)}")
    dt = k.dtype
    if v.dtype != dt:
        raise NexusError(EDTYPE, "cache k and v dtypes differ")
    return _pack_cache(k.data_ptr(), v.data_ptr(), L, npp, P, H, D, BF16 if dt == torch.bfloat16 else _dtype_code(k),
                       cache.v_layout, cache.rope_style, cache.rope_base)


def _vector(name: str, t: torch.Tensor, n):
    """t must be a contiguous int32 vector of n entries (n None: of any)."""
    shape = t.shape
    if t.dtype != _I32 or len(shape) != 1 or (n is not None and shape[0] != n) or not t.is_contiguous():
        raise NexusError(EINVAL, f"{name} must be a contiguous int32 vector" + ("" if n is None else f" of {n}"))


def _page_rows(maps: torch.Tensor, n: int):
    shape = maps.shape
    if maps.dtype != _I32 or len(shape) != 2 or shape[0] != n or not maps.is_contiguous():
        raise NexusError(EINVAL, "maps must be a contiguous int32 [n_seqs][stride] device tensor")


def batch_pages(maps: torch.Tensor, cached: torch.Tensor, fresh: torch.Tensor, free_pages: torch.Tensor,
                n_free: torch.Tensor, max_tokens: int, out: BatchRows | None = None) -> BatchRows:
    """Lays a round out: ``fresh`` tokens of sequences that hold ``cached`` ones (device int32 [n_seqs]) get rows,
    pages from the end of ``free_pages``' first ``n_free`` entries into their rows of ``maps`` [n_seqs][stride],
    positions and slots.  ``out`` may hold the tensors to write (a captured round)."""
    n = cached.shape[0] if cached.dim() == 1 else -1
    _vector("cached", cached, n)
    _vector("fresh", fresh, n)
    _vector("free_pages", free_pages, None)
    _vector("n_free", n_free, 1)
    _page_rows(maps, n)
    dev = _current_of(maps, cached, fresh, free_pages, n_free)
    if dev < 0:
        _here(maps=maps, cached=cached, fresh=fresh, free_pages=free_pages, n_free=n_free)
    if max_tokens >> 30:
        if max_tokens > 1 << 30:
            raise NexusError(ERANGE, "max_tokens must be at most 2^30")
        max_tokens = _int32(max_tokens)
    if out is None:
        out = BatchRows.empty(n, max(0, max_tokens), maps.device)
    else:
        for name, size in (("q_start", n + 1), ("seq_len", n), ("pos", max_tokens), ("slot", max_tokens), ("n_left", 1)):
            _vector(name, getattr(out, name), size)
        if not _all_here(out.q_start, out.seq_len, out.pos, out.slot, out.n_left):
            _here(q_start=out.q_start, seq_len=out.seq_len, pos=out.pos, slot=out.slot, n_left=out.n_left)
    # (a list of no entries has no address, and none of it is read: any will do)
    st = lib().nexus_batch_pages(cached.data_ptr(), fresh.data_ptr(), n, free_pages.data_ptr() or n_free.data_ptr(),
                                 n_free.data_ptr(), free_pages.shape[0], maps.data_ptr(), maps.shape[1], max_tokens,
                                 out.q_start.data_ptr(), out.seq_len.data_ptr(), out.pos.data_ptr(),
                                 out.slot.data_ptr(), out.n_left.data_ptr(), _stream_of(dev))
    if st != OK:
        raise NexusError(st, "nexus_batch_pages")
    return out


def _row_stride(name: str, x: torch.Tensor, rows: int, heads, dim: int, dtype) -> int:
    """Elements between the rows of x [rows][heads][dim], whose heads follow one another."""
    shape = x.shape
    if len(shape) != 3 or shape[0] != rows or (heads is not None and shape[1] != heads) or shape[2] != dim:
        raise NexusError(ESHAPE, f"{name} must be [rows][heads][D] with the cache's heads and D, got {tuple(shape)}")
    if x.dtype != dtype:
        raise NexusError(EDTYPE, f"{name}'s dtype differs from the cache's")
    st = x.stride()
    if st[2] != 1 or (st[1] != dim and shape[1] > 1):
        raise NexusError(EINVAL, f"the heads of a row of {name} must be contiguous")
    return st[0] if rows > 1 else shape[1] * dim


def norm_rope_append(cache: PagedKVCache, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                     pos: torch.Tensor, slot: torch.Tensor, q_weight: torch.Tensor | None = None,
                     k_weight: torch.Tensor | None = None, eps: float = 0.0,
                     out: torch.Tensor | None = None) -> torch.Tensor:
    """The rows of one layer: q [rows][n_q_heads][D], k and v [rows][n_kv_heads][D], which may be parts of one
    projection's rows, with ``pos`` and ``slot`` [rows] of batch_pages.  Heads of q and k are normalised where eps > 0
    (weights fp32 [D]) and rotated to their positions; keys and values go to their slots, queries to the tensor that
    is returned (rows without a slot are not written; ``out`` may be q)."""
    if layer >> 31:
        layer = _int32(layer)
    desc, ck, cv = _descriptor(cache), cache.k, cache.v
    dt, hkv, dim = ck.dtype, ck.shape[2], ck.shape[4]
    rows = q.shape[0]
    qs, ks, vs = (_row_stride("q", q, rows, None, dim, dt), _row_stride("k", k, rows, hkv, dim, dt),
                  _row_stride("v", v, rows, hkv, dim, dt))
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None and (w.dtype != torch.float32 or w.shape != (dim,) or not w.is_contiguous()):
            raise NexusError(EINVAL, f"{name} must be a contiguous fp32 vector of head_dim")
    _vector("pos", pos, rows)
    _vector("slot", slot, rows)
    if out is not None and (out.shape != q.shape or out.dtype != dt or not out.is_contiguous()):
        raise NexusError(EINVAL, "out must be contiguous, shaped and typed like q")
    dev = _current_of(ck, cv, q, k, v, out, q_weight, k_weight, pos, slot)
    if dev < 0:
        _here(cache_k=ck, cache_v=cv, q=q, k=k, v=v, out=out, q_weight=q_weight, k_weight=k_weight, pos=pos, slot=slot)
    if out is None:
        out = torch.empty(q.shape, dtype=dt, device=q.device)
    st = lib().nexus_norm_rope_append(desc, layer, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, rows,
                                      q.shape[1], _ptr(q_weight), _ptr(k_weight), eps, pos.data_ptr(),
                                      slot.data_ptr(), out.data_ptr(), _stream_of(dev))
    if st != OK:
        raise NexusError(st, "nexus_norm_rope_append")
    return out


def _window_operands(q, cache, maps, q_start, seq_len, out, workspace):
    """Checks the operands of a windowed launch (q_start None: a row a sequence); returns the cache's descriptor, out,
    n_seqs and the stream."""
    desc, k = _descriptor(cache), cache.k
    shape = q.shape
    if len(shape) != 3 or shape[2] != k.shape[4]:
        raise NexusError(ESHAPE, "q must be [rows][n_q_heads][D] with the cache's D")
    if not q.is_contiguous():
        raise NexusError(EINVAL, "q must be contiguous")
    dt = q.dtype
    if dt != k.dtype:
        raise NexusError(EDTYPE, "q dtype differs from the cache")
    if q_start is None:
        n = shape[0]
    else:
        n = seq_len.shape[0] if seq_len.dim() == 1 else -1
        _vector("q_start", q_start, n + 1)
    _vector("seq_len", seq_len, n)
    _page_rows(maps, n)
    if out is not None and (out.shape != shape or out.dtype != dt or not out.is_contiguous()):
        raise NexusError(EINVAL, "out must be contiguous, shaped and typed like q")
    if workspace is not None and not workspace.is_contiguous():
        raise NexusError(EINVAL, "workspace must be contiguous")
    dev = _current_of(k, cache.v, q, maps, seq_len, q_start, out, workspace)
    if dev < 0:
        _here(cache_k=k, cache_v=cache.v, q=q, maps=maps, seq_len=seq_len, q_start=q_start, out=out,
              workspace=workspace)
    return desc, torch.empty_like(q) if out is None else out, n, _stream_of(dev)


def _window_call(call, need, args, q: torch.Tensor, workspace, stream, what: str):
    """call(*args, workspace, bytes, stream); need() are the bytes of a workspace that the caller has not given, asked for
    only where the call says that it needs one (nothing is enqueued then)."""
    if workspace is None:
        st = call(*args, 0, 0, stream)
        if st == EWORKSPACE:
            workspace = torch.empty(need(), dtype=torch.uint8, device=q.device)     # held until the call returns
            st = call(*args, workspace.data_ptr(), workspace.numel(), stream)
    else:
        st = call(*args, workspace.data_ptr(), workspace.numel() * workspace.element_size(), stream)
    if st != OK:
        raise NexusError(st, what)


def window_attn(q: torch.Tensor, cache: PagedKVCache, maps: torch.Tensor, q_start: torch.Tensor,
                seq_len: torch.Tensor, max_seq_len: int, window: int, n_sink: int, layer: int, softcap: float = 0.0,
                v_layout: int | None = None, scale: float = 0.0, out: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None):
    """Attention of a ragged batch in a sliding window with ``n_sink`` first tokens in sight: rows q_start[b] ..
    q_start[b + 1] - 1 of q [rows][n_q_heads][D] are the last ones of sequence b, of seq_len[b] tokens behind row b of
    ``maps`` (device int32 tensors).  Rows of no sequence are left as they are in out (without ``out``: undefined)."""
    if (window | n_sink | max_seq_len | layer) >> 31:          # (a call of _int32 for each costs 0.3 us of host time)
        window, n_sink, max_seq_len, layer = map(_int32, (window, n_sink, max_seq_len, layer))
    L = lib()
    c, out, n, stream = _window_operands(q, cache, maps, q_start, seq_len, out, workspace)
    rows, hq, _ = q.shape
    _window_call(L.nexus_window_attn,
                 lambda: L.nexus_window_attn_workspace(rows, hq, c, n, max_seq_len, window, n_sink),
                 (q.data_ptr(), rows, hq, c, maps.data_ptr(), maps.shape[1], q_start.data_ptr(), seq_len.data_ptr(), n,
                  max_seq_len, window, n_sink, layer, softcap, cache.v_layout if v_layout is None else v_layout, scale,
                  out.data_ptr()), q, workspace, stream, "nexus_window_attn")
    return out


def window_attn_workspace_bytes(cache: PagedKVCache, n_rows: int, n_q_heads: int, n_seqs: int, max_seq_len: int,
                                window: int, n_sink: int) -> int:
    n = lib().nexus_window_attn_workspace(_int32(n_rows), _int32(n_q_heads), _descriptor(cache), _int32(n_seqs),
                                          _int32(max_seq_len), _int32(window), _int32(n_sink))
    if n == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_window_attn_workspace")
    return n


def window_decode_attn(q: torch.Tensor, cache: PagedKVCache, maps: torch.Tensor, seq_len: torch.Tensor,
                       max_seq_len: int, window: int, n_sink: int, layer: int, softcap: float = 0.0,
                       v_layout: int | None = None, scale: float = 0.0, out: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None):
    """decode_attn in a sliding window with ``n_sink`` first tokens in sight."""
    if (window | n_sink | max_seq_len | layer) >> 31:          # (a call of _int32 for each costs 0.3 us of host time)
        window, n_sink, max_seq_len, layer = map(_int32, (window, n_sink, max_seq_len, layer))
    L = lib()
    c, out, n, stream = _window_operands(q, cache, maps, None, seq_len, out, workspace)
    hq = q.shape[1]
    _window_call(L.nexus_window_decode_attn,
                 lambda: L.nexus_window_decode_attn_workspace(n, hq, c, max_seq_len, window, n_sink),
                 (q.data_ptr(), n, hq, c, maps.data_ptr(), maps.shape[1], seq_len.data_ptr(), max_seq_len, window,
                  n_sink, layer, softcap, cache.v_layout if v_layout is None else v_layout, scale, out.data_ptr()),
                 q, workspace, stream, "nexus_window_decode_attn")
    return out


def window_decode_attn_workspace_bytes(cache: PagedKVCache, n_seqs: int, n_q_heads: int, max_seq_len: int,
                                       window: int, n_sink: int) -> int:
    n = lib().nexus_window_decode_attn_workspace(_int32(n_seqs), _int32(n_q_heads), _descriptor(cache),
                                                 _int32(max_seq_len), _int32(window), _int32(n_sink))
    if n == (1 << 64) - 1:
        raise NexusError(EINVAL, "nexus_window_decode_attn_workspace")
    return n


def kv_copy_tokens(cache: PagedKVCache, src_map: torch.Tensor, dst_map: torch.Tensor, t0: int,
                   n_tokens: int):
    """Copy logical tokens [t0, t0 + n_tokens) of every layer from the sequence mapped by
    ``src_map`` to the sequence mapped by ``dst_map`` (device int32 maps of equal length)."""
    if src_map.numel() != dst_map.numel():
        raise NexusError(EINVAL, "maps differ in length")
    cc = cache.c()
    _on_device(("cache k", cache.k), ("src_map", src_map), ("dst_map", dst_map))
    _check(lib().nexus_kv_copy_tokens(C.byref(cc), _map_arg(src_map, "src_map"),
                                      _map_arg(dst_map, "dst_map"), src_map.numel(), t0,
                                      n_tokens, _stream()), "nexus_kv_copy_tokens")


def kv_share_prefix(cache: PagedKVCache, src_map: torch.Tensor, dst_map: torch.Tensor,
                    n_tokens: int):
    """Share the first n_tokens tokens of the source with the destination: whole pages by
    reference (dst_map is updated on the device), the partial last page by copy."""
    if src_map.numel() != dst_map.numel():
        raise NexusError(EINVAL, "maps differ in length")
    cc = cache.c()
    _on_device(("cache k", cache.k), ("src_map", src_map), ("dst_map", dst_map))
    _check(lib().nexus_kv_share_prefix(C.byref(cc), _map_arg(src_map, "src_map"),
                                       _map_arg(dst_map, "dst_map"), src_map.numel(), n_tokens,
                                       _stream()), "nexus_kv_share_prefix")


def l0_longest_prefix(tokens, slots):
    """(slot, length) of the slot sharing the longest common prefix with ``tokens`` (host)."""
    import numpy as np
    t = np.ascontiguousarray(np.asarray(tokens, dtype=np.int32))
    n_slots = len(slots)
    stride = max([len(x) for x in slots] + [1])
    arr = np.zeros((max(n_slots, 1), stride), dtype=np.int32)
    lens = np.zeros(max(n_slots, 1), dtype=np.int32)
    for i, x in enumerate(slots):
        arr[i, :len(x)] = x
        lens[i] = len(x)
    P = C.POINTER(C.c_int32)
    slot, mlen = C.c_int32(0), C.c_int32(0)
    _check(lib().nexus_l0_longest_prefix(t.ctypes.data_as(P), t.size, arr.ctypes.data_as(P),
                                         lens.ctypes.data_as(P), n_slots, stride, C.byref(slot),
                                         C.byref(mlen)), "nexus_l0_longest_prefix")
    return slot.value, mlen.value


def slb_quantize(x: torch.Tensor, out=None):
    """x [n][dim] fp32 (device) -> (int8 codes [n][dim], fp32 scales [n]); ``out`` may hold
    preallocated (codes, scales)."""
    if x.dtype != torch.float32 or x.dim() != 2 or not x.is_contiguous() or not x.is_cuda:
        raise NexusError(EINVAL, "x must be a contiguous fp32 [n][dim] device tensor")
    n, dim = x.shape
    if out is None:
        q = torch.empty((n, dim), dtype=torch.int8, device=x.device)
        s = torch.empty((n,), dtype=torch.float32, device=x.device)
    else:
        q, s = out
        if (q.dtype != torch.int8 or tuple(q.shape) != (n, dim) or not q.is_contiguous()
                or s.dtype != torch.float32 or s.numel() != n):
            raise NexusError(EINVAL, "out must be (int8 [n][dim], fp32 [n]) contiguous tensors")
    _on_device(("x", x), ("codes", q), ("scales", s))
    _check(lib().nexus_slb_quantize(_ptr(x), n, dim, _ptr(q), _ptr(s), _stream()),
           "nexus_slb_quantize")
    return q, s


def slb_scan(tools: torch.Tensor, tool_scale: torch.Tensor, queries: torch.Tensor,
             query_scale: torch.Tensor, k: int = 2, tau: float = 0.0136,
             workspace: torch.Tensor | None = None, out=None):
    """Top-k tools per query, the top-two margin and the gate (1 = auto-route).  Returns
    (top_idx [Q][k] int32, top_score [Q][k] fp32, margin [Q] fp32, route [Q] int32)."""
    for t, dt, nd in ((tools, torch.int8, 2), (queries, torch.int8, 2),
                      (tool_scale, torch.float32, 1), (query_scale, torch.float32, 1)):
        if t.dtype != dt or t.dim() != nd or not t.is_contiguous() or not t.is_cuda:
            raise NexusError(EINVAL, "slb_scan: bad operand dtype, shape or device")
    n_tools, dim = tools.shape
    n_q = queries.shape[0]
    if queries.shape[1] != dim or tool_scale.numel() != n_tools or query_scale.numel() != n_q:
        raise NexusError(ESHAPE, "slb_scan: operand shapes disagree")
    dev = _on_device(("tools", tools), ("tool_scale", tool_scale), ("queries", queries),
                     ("query_scale", query_scale), ("workspace", workspace))
    if out is not None:
        _on_device(("tools", tools), *[(f"out[{i}]", t) for i, t in enumerate(out)])
    if out is None:
        out = (torch.empty((n_q, k), dtype=torch.int32, device=dev),
               torch.empty((n_q, k), dtype=torch.float32, device=dev),
               torch.empty((n_q,), dtype=torch.float32, device=dev),
               torch.empty((n_q,), dtype=torch.int32, device=dev))
    ws_bytes = lib().nexus_slb_scan_workspace(n_tools, n_q, dim, k)
    if ws_bytes == (1 << 64) - 1:
        ws_bytes = 0             # invalid arguments: the call itself reports which check failed
    ws = _workspace(ws_bytes, dev, workspace)
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    idx, score, margin, route = out
    _check(lib().nexus_slb_scan(_ptr(tools), _ptr(tool_scale), n_tools, _ptr(queries),
                                _ptr(query_scale), n_q, dim, k, tau, _ptr(idx), _ptr(score),
                                _ptr(margin), _ptr(route), _ptr(ws), nbytes, _stream()),
           "nexus_slb_scan")
    return out


def redecode_len(S: int, n_past: int, M: int = 256, r_base_pct: int = 5, K: int = 4) -> int:
    r = lib().nexus_redecode_len(S, n_past, M, r_base_pct, K)
    if r < 0:
        raise NexusError(EINVAL, "nexus_redecode_len")
    return r


def check_page_table(host_map, n_phys_pages: int) -> None:
    import numpy as np
    a = np.ascontiguousarray(np.asarray(host_map, dtype=np.int32))
    _check(lib().nexus_check_page_table(a.ctypes.data_as(C.POINTER(C.c_int32)), a.size,
                                        n_phys_pages), "nexus_check_page_table")


def calib_copy(src: torch.Tensor, dst: torch.Tensor):
    """Device copy of src's bytes into dst (measurement helper: the HBM read + write ceiling)."""
    _on_device(("src", src), ("dst", dst))
    n = src.numel() * src.element_size()
    if not (src.is_contiguous() and dst.is_contiguous()) or dst.numel() * dst.element_size() < n:
        raise NexusError(EINVAL, "calib_copy: contiguous src, and dst at least as large")
    _check(lib().nexus_calib_copy(_ptr(src), _ptr(dst), n, _stream()), "nexus_calib_copy")


def calib_lds_dma(src: torch.Tensor):
    """Stream src's bytes into LDS with LDS DMA loads (measurement helper: the reference for the
    memory counters' reading of the attention kernels' loads)."""
    _on_device(("src", src))
    n = src.numel() * src.element_size()
    if not src.is_contiguous() or n == 0 or n % 16384:
        raise NexusError(EINVAL, "calib_lds_dma: contiguous src of a multiple of 16384 bytes")
    _check(lib().nexus_calib_lds_dma(_ptr(src), n, _stream()), "nexus_calib_lds_dma")


def calib_mfma_bf16(iters: int, sink: torch.Tensor) -> float:
    """Enqueue the bf16 MFMA ceiling kernel; returns the matrix FLOPs it performs."""
    _on_device(("sink", sink))
    if sink.dtype != torch.float32 or sink.numel() < 512:
        raise NexusError(EINVAL, "calib_mfma_bf16: sink must hold 512 fp32 values")
    fl = C.c_double(0.0)
    _check(lib().nexus_calib_mfma_bf16(iters, _ptr(sink), C.byref(fl), _stream()),
           "nexus_calib_mfma_bf16")
    return fl.value
