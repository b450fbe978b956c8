"""ctypes binding of libsttm.so: same names as include/sttm.h, argument marshalling only.

Device buffers are torch tensors (torch is used for device memory and streams, nothing else); every
step of the path runs inside the library's HIP kernels.  There is no fallback: if the shared library
is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np
import torch  # noqa: F401  -- first, so that libsttm.so binds to the HIP runtime torch has already loaded

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsttm.so")

STTM_OK = 0
STTM_ERR_NULL, STTM_ERR_SHAPE, STTM_ERR_DTYPE, STTM_ERR_ARG = 1, 2, 3, 4
STTM_ERR_WORKSPACE, STTM_ERR_STATE, STTM_ERR_CAPACITY, STTM_ERR_HIP = 5, 6, 7, 8
STTM_F32, STTM_BF16, STTM_F16 = 0, 1, 2
STTM_STAGE_SPATIAL, STTM_STAGE_TEMPORAL = 0, 1
STTM_TBL_CHILD_SIM, STTM_TBL_MIN_SIM, STTM_TBL_NORM2 = 0, 1, 2
STTM_TBL_PAIR_SIM, STTM_TBL_BEST_SIM, STTM_TBL_PARENT = 3, 4, 5

EXPORTS = [
    "sttm_create", "sttm_destroy", "sttm_last_error", "sttm_nodes_per_frame", "sttm_node_index",
    "sttm_workspace_bytes", "sttm_set_workspace", "sttm_spatial_stats", "sttm_spatial_quadtree",
    "sttm_temporal_stats", "sttm_temporal_merge", "sttm_budget_threshold", "sttm_reduce", "sttm_export",
    "sttm_profile_enable", "sttm_profile_read", "sttm_set_match_mode", "sttm_set_output_order", "sttm_positions",
    "sttm_set_cell_dots", "sttm_invalidate", "sttm_reduce_noalloc", "sttm_reduce_noalloc_max_bytes",
    "sttm_reduce_noalloc_bytes", "sttm_qk_norm_rope", "sttm_paged_attention", "sttm_paged_attention_workspace_bytes",
    "sttm_cache_evict", "sttm_cache_evict_workspace_bytes",
]
STTM_MATCH_FIRST_PASSING, STTM_MATCH_TOPLEFT_ONLY, STTM_MATCH_MOST_SIMILAR = 0, 1, 2
STTM_ORDER_RASTER, STTM_ORDER_ZSCAN = 0, 1
STTM_KERNEL_PYRAMID_STATS, STTM_KERNEL_TEMPORAL_DOTS, STTM_KERNEL_REDUCE_GATHER = 0, 1, 2


class _CacheStruct(C.Structure):
    """sttm_cache"""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("dtype", C.c_int), ("kv_heads", C.c_int), ("head_dim", C.c_int),
                ("page_size", C.c_int), ("pages", C.c_int64), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("token_stride", C.c_int64)]


class _SequencesStruct(C.Structure):
    """sttm_sequences"""
    _fields_ = [("block_table", C.c_void_p), ("lengths", C.c_void_p), ("table_stride", C.c_int64), ("batch", C.c_int),
                ("max_pages", C.c_int), ("max_len", C.c_int)]


class _RopeStruct(C.Structure):
    """sttm_rope"""
    _fields_ = [("positions", C.c_void_p), ("inv_freq", C.c_void_p), ("pos_stride", C.c_int64), ("sections", C.c_int * 3),
                ("pos_float", C.c_int), ("interleaved", C.c_int)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2507_07990_amd.build` "
            "(there is no CPU fallback)")
    return _declare(C.CDLL(LIB_PATH))


def _declare(lib: C.CDLL) -> C.CDLL:
    vp, i, i64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
    lib.sttm_create.argtypes = [C.POINTER(vp), i, vp]
    lib.sttm_destroy.argtypes = [vp]
    lib.sttm_last_error.argtypes = [vp]
    lib.sttm_last_error.restype = C.c_char_p
    lib.sttm_nodes_per_frame.argtypes = [i, i, i]
    lib.sttm_node_index.argtypes = [i, i, i, i, i, i]
    lib.sttm_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
    lib.sttm_workspace_bytes.restype = sz
    lib.sttm_set_workspace.argtypes = [vp, vp, sz]
    lib.sttm_spatial_stats.argtypes = [vp, vp, i, i, i, i, i, i, i]
    lib.sttm_spatial_quadtree.argtypes = [vp, vp, i, i, i, i, i, i, i, C.POINTER(C.c_float), vp, vp]
    lib.sttm_temporal_stats.argtypes = [vp, vp, vp, vp]
    lib.sttm_temporal_merge.argtypes = [vp, vp, vp, vp, C.POINTER(C.c_float), vp]
    lib.sttm_budget_threshold.argtypes = [vp, i, C.POINTER(C.c_double), C.POINTER(C.c_float)]
    lib.sttm_reduce.argtypes = [vp, vp, vp, vp, vp, i, i64, vp, vp, vp, vp, C.POINTER(i64)]
    lib.sttm_export.argtypes = [vp, i, vp, sz]
    lib.sttm_profile_enable.argtypes = [vp, i]
    lib.sttm_profile_read.argtypes = [vp, i, C.POINTER(C.c_double), C.POINTER(i64)]
    lib.sttm_set_match_mode.argtypes = [vp, i]
    lib.sttm_set_output_order.argtypes = [vp, i]
    lib.sttm_set_cell_dots.argtypes = [vp, i]
    lib.sttm_invalidate.argtypes = [vp]
    lib.sttm_reduce_noalloc.argtypes = [vp, vp, i, i, i, i, i, i, vp, i, i64, vp, vp, vp, vp]
    lib.sttm_reduce_noalloc_max_bytes.argtypes = []
    lib.sttm_reduce_noalloc_max_bytes.restype = sz
    lib.sttm_reduce_noalloc_bytes.argtypes = [i, i, i, i, i, i]
    lib.sttm_reduce_noalloc_bytes.restype = sz
    lib.sttm_positions.argtypes = [vp, vp, vp, vp, vp, i64, vp, vp, vp, vp]
    f, cache, seqs, rope = C.c_float, C.POINTER(_CacheStruct), C.POINTER(_SequencesStruct), C.POINTER(_RopeStruct)
    lib.sttm_qk_norm_rope.argtypes = [vp, i, i64, i, i, i, vp, i64, vp, i64, vp, i64, vp, vp, f, rope, vp, i64, vp, i64, cache, vp]
    lib.sttm_paged_attention.argtypes = [vp, cache, seqs, i, f, vp, i64, vp, vp, vp, i64, vp, i64, vp, vp, sz]
    lib.sttm_paged_attention_workspace_bytes.argtypes = [cache, seqs, i, i]
    lib.sttm_paged_attention_workspace_bytes.restype = sz
    lib.sttm_cache_evict.argtypes = [vp, cache, seqs, vp, vp, i, i, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz]
    lib.sttm_cache_evict_workspace_bytes.argtypes = [cache, seqs]
    lib.sttm_cache_evict_workspace_bytes.restype = sz
    return lib


_lib = _load()


class SttmError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"sttm status {code}: {msg}")
        self.code = code


def sttm_nodes_per_frame(H: int, W: int, root_grid: int = 1) -> int:
    return int(_lib.sttm_nodes_per_frame(H, W, root_grid))


def sttm_node_index(H: int, W: int, root_grid: int, level: int, by: int, bx: int) -> int:
    return int(_lib.sttm_node_index(H, W, root_grid, level, by, bx))


def sttm_workspace_bytes(B, T, H, W, D, dtype, root_grid=1) -> int:
    return int(_lib.sttm_workspace_bytes(B, T, H, W, D, dtype, root_grid))


def sttm_reduce_noalloc_max_bytes() -> int:
    return int(_lib.sttm_reduce_noalloc_max_bytes())


def sttm_reduce_noalloc_bytes(B, T, H, W, D, dtype) -> int:
    return int(_lib.sttm_reduce_noalloc_bytes(B, T, H, W, D, dtype))


_DTYPES = {torch.float32: STTM_F32, torch.bfloat16: STTM_BF16, torch.float16: STTM_F16}


def _expect(ok: bool, code: int, msg: str):
    if not ok:
        raise SttmError(code, msg)


class PagedCache:
    """sttm_cache: keys and values, tensors [pages, kv_heads, page_size, head_dim] of one type and one set of strides (the
    last one 1; e.g. two views of one buffer, or [pages, page_size, kv_heads, head_dim] with the middle axes exchanged)."""

    def __init__(self, k, v):
        _expect(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride() and k.stride(3) == 1, STTM_ERR_SHAPE,
                "k and v must be [pages, kv_heads, page_size, head_dim] with the same strides, the last one 1")
        _expect(k.dtype == v.dtype and k.dtype in _DTYPES, STTM_ERR_DTYPE, "k and v must be of one type, float32, bfloat16 or float16")
        _expect(k.device == v.device, STTM_ERR_ARG, "k and v must be on one device")
        self.k, self.v, self.dtype, self.device = k, v, k.dtype, k.get_device()   # (the tensors live as long as this)
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        strides = [st if n > 1 else 0 for n, st in zip(k.shape, k.stride())]   # (the stride of a single entry means nothing)
        self.struct = _CacheStruct(_ptr(k), _ptr(v), _DTYPES[k.dtype], self.kv_heads, self.head_dim, self.page_size, self.pages,
                                   strides[0], strides[1], strides[2] or self.head_dim)
        self.ref = C.byref(self.struct)


class Sequences:
    """sttm_sequences: block_table int32 [batch, max_pages] (rows any stride apart), lengths int32 [batch]; no length is above
    max_len (default: the slots of a table row)."""

    def __init__(self, block_table, lengths, max_len: Optional[int] = None):
        _expect(block_table.dim() == 2 and lengths.dim() == 1 and block_table.shape[0] == lengths.shape[0], STTM_ERR_SHAPE,
                "block_table must be [batch, max_pages], lengths [batch]")
        _expect(block_table.dtype == torch.int32 and lengths.dtype == torch.int32, STTM_ERR_DTYPE, "block_table and lengths must be int32")
        batch, pages = block_table.shape
        _expect((pages <= 1 or block_table.stride(1) == 1) and (batch <= 1 or lengths.stride(0) == 1), STTM_ERR_SHAPE,
                "the rows of block_table and lengths must be contiguous")
        _expect(block_table.device == lengths.device, STTM_ERR_ARG, "block_table and lengths must be on one device")
        _expect(max_len is None or max_len >= 0, STTM_ERR_SHAPE, "max_len must not be negative")
        self.block_table, self.lengths, self.batch, self.device = block_table, lengths, batch, lengths.get_device()
        self.max_pages, self.max_len = pages, 2**31 - 1 if max_len is None else min(int(max_len), 2**31 - 1)
        self.struct = _SequencesStruct(_ptr(block_table), _ptr(lengths), block_table.stride(0) if batch > 1 else pages, batch, pages,
                                       self.max_len)
        self.ref = C.byref(self.struct)


class Rope:
    """sttm_rope: positions int32 or float32 [n, axes or more] (or [n]: one axis), inv_freq float32 [pairs], sections: pairs
    for each axis (default: all on the first)."""

    def __init__(self, positions, inv_freq, sections: Optional[Sequence[int]] = None, interleaved: bool = False):
        _expect(positions.dtype in (torch.int32, torch.float32) and inv_freq.dtype == torch.float32, STTM_ERR_DTYPE,
                "positions must be int32 or float32, inv_freq float32")
        _expect(inv_freq.dim() == 1 and (inv_freq.numel() <= 1 or inv_freq.stride(0) == 1), STTM_ERR_SHAPE, "inv_freq must be [pairs], contiguous")
        if positions.dim() == 1:
            positions = positions[:, None]
        _expect(positions.dim() == 2 and (positions.shape[1] <= 1 or positions.stride(1) == 1), STTM_ERR_SHAPE,
                "positions must be [n] or [n, axes] with contiguous rows")
        parts = [inv_freq.numel()] if sections is None else [int(x) for x in sections]
        _expect(1 <= len(parts) <= min(3, max(1, positions.shape[1])) and sum(parts) == inv_freq.numel() and min(parts) >= 0, STTM_ERR_SHAPE,
                "sections: one to three numbers of pairs that add up to inv_freq's, no more of them than positions has axes")
        _expect(positions.device == inv_freq.device, STTM_ERR_ARG, "positions and inv_freq must be on one device")
        self.positions, self.inv_freq, self.device, self.n = positions, inv_freq, inv_freq.get_device(), positions.shape[0]
        stride = positions.stride(0) if self.n > 1 else positions.shape[1]
        self.struct = _RopeStruct(_ptr(positions), _ptr(inv_freq), stride, (C.c_int * 3)(*parts, *[0] * (3 - len(parts))),
                                  int(positions.dtype == torch.float32), int(interleaved))
        self.ref = C.byref(self.struct)


def sttm_paged_attention_workspace_bytes(cache: PagedCache, sequences: Sequences, q_heads: int, weights: bool = False) -> int:
    return int(_lib.sttm_paged_attention_workspace_bytes(cache.struct, sequences.struct, q_heads, int(weights)))


def sttm_cache_evict_workspace_bytes(cache: PagedCache, sequences: Sequences) -> int:
    return int(_lib.sttm_cache_evict_workspace_bytes(cache.struct, sequences.struct))


# The checks below run on every call of a decoding loop: a handful of comparisons, messages only where one fails.

def _rows(t, name: str, n: int, heads: int, d: int, dtype, device: int) -> int:
    """The elements between the rows of t [n, heads, d], whose heads lie one after the other."""
    stride = t.stride()
    if t.shape != (n, heads, d) or stride[2] != 1 or (stride[1] != d and heads != 1):
        raise SttmError(STTM_ERR_SHAPE, f"{name} must be [{n}, {heads}, {d}], the heads of a row one after the other")
    if t.dtype is not dtype or t.get_device() != device:
        raise SttmError(STTM_ERR_DTYPE, f"{name} must be of the type and on the device of the others")
    return stride[0] if n > 1 else heads * d


def _table(t, name: str, dtype, shape, device: int) -> Optional[int]:
    """The address of t [batch, kv_heads, slots], contiguous, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device:
        raise SttmError(STTM_ERR_DTYPE, f"{name} must be {dtype} on the cache's device")
    if t.shape != shape or not t.is_contiguous():
        raise SttmError(STTM_ERR_SHAPE, f"{name} must be [batch, kv_heads, slots], contiguous, with as many slots as the other tables")
    return t.data_ptr()


def _vector(t, name: str, dtype, n: int, device: int) -> Optional[int]:
    """The address of t, n entries, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device:
        raise SttmError(STTM_ERR_DTYPE, f"{name} must be {dtype} on the device of the others")
    if t.numel() != n or not t.is_contiguous():
        raise SttmError(STTM_ERR_SHAPE, f"{name} must have {n} entries, contiguous")
    return t.data_ptr()


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _farr(vals: Optional[Sequence[float]], n: int):
    if vals is None:
        return None
    a = np.broadcast_to(np.asarray(vals, dtype=np.float32), (n,))
    return (C.c_float * n)(*[float(v) for v in a])


class Sttm:
    """One library context on one device / stream.  Methods mirror the C entry points."""

    def __init__(self, device: int = 0, stream_ptr: Optional[int] = None):
        import torch
        if stream_ptr is None:
            stream_ptr = torch.cuda.current_stream(device).cuda_stream
        self._h = C.c_void_p()
        rc = _lib.sttm_create(C.byref(self._h), device, C.c_void_p(stream_ptr))
        if rc != STTM_OK:
            raise SttmError(rc, "sttm_create failed")
        self.device = self._device_index = device
        self._ws = None
        self.shape = None

    def close(self):
        if self._h:
            _lib.sttm_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc != STTM_OK:
            raise SttmError(rc, _lib.sttm_last_error(self._h).decode())

    # -- workspace ------------------------------------------------------------------------------
    def sttm_set_workspace(self, ws_tensor):
        self._ws = ws_tensor
        self._check(_lib.sttm_set_workspace(self._h, _ptr(ws_tensor), ws_tensor.numel() * ws_tensor.element_size()))

    def ensure_workspace(self, B, T, H, W, D, dtype, root_grid=1):
        import torch
        need = sttm_workspace_bytes(B, T, H, W, D, dtype, root_grid)
        if need == 0:
            raise SttmError(STTM_ERR_SHAPE, "invalid shape")
        if self._ws is None or self._ws.numel() < need:
            self.sttm_set_workspace(torch.empty(need, dtype=torch.uint8, device=f"cuda:{self.device}"))

    # -- stages -----------------------------------------------------------------------------------
    def sttm_spatial_stats(self, feats, dtype, B, T, H, W, D, root_grid=1):
        self._check(_lib.sttm_spatial_stats(self._h, _ptr(feats), dtype, B, T, H, W, D, root_grid))
        self.shape = (B, T, H, W, D, dtype, root_grid)

    def sttm_spatial_quadtree(self, feats, dtype, B, T, H, W, D, root_grid, tau_s, node_map, node_level=None):
        self._check(_lib.sttm_spatial_quadtree(self._h, _ptr(feats), dtype, B, T, H, W, D, root_grid,
                                               _farr(tau_s, B), _ptr(node_map), _ptr(node_level)))
        self.shape = (B, T, H, W, D, dtype, root_grid)

    def sttm_temporal_stats(self, feats, node_map, node_level=None):
        self._check(_lib.sttm_temporal_stats(self._h, _ptr(feats), _ptr(node_map), _ptr(node_level)))

    def sttm_temporal_merge(self, feats, node_map, node_level, tau_t, cluster_ids):
        B = self.shape[0]
        self._check(_lib.sttm_temporal_merge(self._h, _ptr(feats), _ptr(node_map), _ptr(node_level),
                                             _farr(tau_t, B), _ptr(cluster_ids)))

    def sttm_budget_threshold(self, stage, target_keep, want_tau=True):
        B = self.shape[0]
        keep = np.broadcast_to(np.asarray(target_keep, dtype=np.float64), (B,))
        karr = (C.c_double * B)(*[float(v) for v in keep])
        out = (C.c_float * B)() if want_tau else None
        self._check(_lib.sttm_budget_threshold(self._h, stage, karr, out))
        return np.array(list(out), dtype=np.float32) if want_tau else None

    def sttm_reduce(self, feats, cluster_ids, node_map, node_level, out_dtype, capacity, merged, counts, out_ids,
                    offsets, want_n=True):
        n = C.c_int64(-1)
        rc = _lib.sttm_reduce(self._h, _ptr(feats), _ptr(cluster_ids), _ptr(node_map), _ptr(node_level), out_dtype,
                              capacity, _ptr(merged), _ptr(counts), _ptr(out_ids), _ptr(offsets),
                              C.byref(n) if want_n else None)
        self._check(rc)
        return int(n.value) if want_n else None

    def sttm_set_match_mode(self, mode: int):
        self._check(_lib.sttm_set_match_mode(self._h, mode))

    def sttm_set_output_order(self, order: int):
        self._check(_lib.sttm_set_output_order(self._h, order))

    def sttm_reduce_noalloc(self, feats, dtype, B, T, H, W, D, cluster_ids, out_dtype, capacity, merged, counts,
                            out_ids, offsets):
        self._check(_lib.sttm_reduce_noalloc(self._h, _ptr(feats), dtype, B, T, H, W, D, _ptr(cluster_ids), out_dtype,
                                             capacity, _ptr(merged), _ptr(counts), _ptr(out_ids), _ptr(offsets)))

    def sttm_invalidate(self):
        self._check(_lib.sttm_invalidate(self._h))

    def sttm_set_cell_dots(self, on: int):
        self._check(_lib.sttm_set_cell_dots(self._h, on))

    def sttm_positions(self, cluster_ids, node_map, node_level, offsets, capacity, survived=None, reassigned=None,
                       merged_pos=None, root_tyxl=None):
        self._check(_lib.sttm_positions(self._h, _ptr(cluster_ids), _ptr(node_map), _ptr(node_level), _ptr(offsets),
                                        capacity,
                                        _ptr(survived), _ptr(reassigned), _ptr(merged_pos), _ptr(root_tyxl)))

    # -- the reduced sequence in a model: a paged cache of keys and values -----------------------------
    def _on_device(self, device: int):
        if device != self._device_index:
            raise SttmError(STTM_ERR_ARG, "the tensors must be on the context's device")

    def _scratch(self, t, device: int):
        if t is None:
            return None, 0
        if t.get_device() != device:
            raise SttmError(STTM_ERR_ARG, "the workspace must be on the tensors' device")
        if not t.is_contiguous():
            raise SttmError(STTM_ERR_SHAPE, "the workspace must be contiguous")
        return t.data_ptr(), t.nbytes

    def sttm_qk_norm_rope(self, q, k, v, q_out, k_out=None, cache: Optional[PagedCache] = None, slots=None, q_weight=None,
                          k_weight=None, eps: float = 1e-6, rope: Optional[Rope] = None):
        """q [n, q_heads, d], k and v [n, kv_heads, d] (views of one projection's output will do); q_out, k_out of the same
        shapes (or q and k themselves). cache, slots int64 [n]: where keys and values go."""
        if q.dim() != 3 or k.dim() != 3:
            raise SttmError(STTM_ERR_SHAPE, "q and k must be [n, heads, head_dim]")
        n, q_heads, d = q.shape
        kv_heads, dtype, dev = k.shape[1], q.dtype, q.get_device()
        self._on_device(dev)
        if dtype not in _DTYPES:
            raise SttmError(STTM_ERR_DTYPE, "float32, bfloat16 or float16")
        qs, ks = _rows(q, "q", n, q_heads, d, dtype, dev), _rows(k, "k", n, kv_heads, d, dtype, dev)
        qos = _rows(q_out, "q_out", n, q_heads, d, dtype, dev)
        vs = kos = 0
        v_at = k_out_at = slots_at = None
        if k_out is not None:
            kos, k_out_at = _rows(k_out, "k_out", n, kv_heads, d, dtype, dev), k_out.data_ptr()
        if cache is not None:
            if slots is None or v is None or cache.device != dev:
                raise SttmError(STTM_ERR_ARG, "a cache on the same device, values, and the rows' slots in it")
            vs, v_at = _rows(v, "v", n, kv_heads, d, dtype, dev), v.data_ptr()
            slots_at = _vector(slots, "slots", torch.int64, n, dev)
        if rope is not None and (rope.n != n or rope.device != dev):
            raise SttmError(STTM_ERR_SHAPE, "the rotation must have a position for each row, on the same device")
        rc = _lib.sttm_qk_norm_rope(self._h, _DTYPES[dtype], n, q_heads, kv_heads, d, q.data_ptr(), qs, k.data_ptr(), ks, v_at, vs,
                                    _vector(q_weight, "q_weight", dtype, d, dev), _vector(k_weight, "k_weight", dtype, d, dev), eps,
                                    rope.ref if rope is not None else None, q_out.data_ptr(), qos, k_out_at, kos,
                                    cache.ref if cache is not None else None, slots_at)
        if rc != STTM_OK:
            self._check(rc)

    def sttm_paged_attention(self, q, cache: PagedCache, sequences: Sequences, out, scale: float, key_bias=None, weights_in=None,
                             weights_out=None, lse=None, workspace=None):
        """q, out [batch, q_heads, d]; key_bias, weights_in, weights_out float32 [batch, kv_heads, slots]; lse float32
        [batch, q_heads]; workspace: sttm_paged_attention_workspace_bytes() bytes."""
        batch, dev, d = sequences.batch, cache.device, cache.head_dim
        self._on_device(dev)
        if sequences.device != dev or q.dim() != 3:
            raise SttmError(STTM_ERR_ARG, "sequences on the cache's device, q [batch, q_heads, head_dim]")
        q_heads = q.shape[1]
        qs, os_ = _rows(q, "q", batch, q_heads, d, cache.dtype, dev), _rows(out, "out", batch, q_heads, d, cache.dtype, dev)
        slots, bias_at, in_at, out_at = 0, None, None, None
        first = key_bias if key_bias is not None else weights_out if weights_out is not None else weights_in
        if first is not None:
            slots = first.shape[-1]
            shape = (batch, cache.kv_heads, slots)
            bias_at = _table(key_bias, "key_bias", torch.float32, shape, dev)
            in_at = _table(weights_in, "weights_in", torch.float32, shape, dev)
            out_at = _table(weights_out, "weights_out", torch.float32, shape, dev)
        ws, size = self._scratch(workspace, dev)
        rc = _lib.sttm_paged_attention(self._h, cache.ref, sequences.ref, q_heads, scale, q.data_ptr(), qs, bias_at, in_at, out_at,
                                       slots, out.data_ptr(), os_, _vector(lse, "lse", torch.float32, batch * q_heads, dev), ws, size)
        if rc != STTM_OK:
            self._check(rc)

    def sttm_cache_evict(self, cache: PagedCache, sequences: Sequences, keep, lengths_out, weights_in, weights_out, ids_in, ids_out,
                         total=None, sink: int = 0, recent: int = 0, bias_in=None, bias_out=None, workspace=None):
        """keep, total, lengths_out int32 [batch]; weights_*, bias_* float32 and ids_* int32 [batch, kv_heads, slots];
        workspace: sttm_cache_evict_workspace_bytes() bytes."""
        batch, dev, f32, i32 = sequences.batch, cache.device, torch.float32, torch.int32
        self._on_device(dev)
        if sequences.device != dev:
            raise SttmError(STTM_ERR_ARG, "sequences on the cache's device")
        shape = (batch, cache.kv_heads, weights_in.shape[-1])
        ws, size = self._scratch(workspace, dev)
        rc = _lib.sttm_cache_evict(self._h, cache.ref, sequences.ref, _vector(keep, "keep", i32, batch, dev),
                                   _vector(total, "total", i32, batch, dev), sink, recent, shape[2],
                                   _table(weights_in, "weights_in", f32, shape, dev), _table(weights_out, "weights_out", f32, shape, dev),
                                   _table(ids_in, "ids_in", i32, shape, dev), _table(ids_out, "ids_out", i32, shape, dev),
                                   _table(bias_in, "bias_in", f32, shape, dev), _table(bias_out, "bias_out", f32, shape, dev),
                                   _vector(lengths_out, "lengths_out", i32, batch, dev), ws, size)
        if rc != STTM_OK:
            self._check(rc)

    def sttm_export(self, table, dst):
        self._check(_lib.sttm_export(self._h, table, _ptr(dst), dst.numel() * dst.element_size()))

    def sttm_profile_enable(self, every):
        """every: False / 0 = off, True / 1 = every launch, n = every n-th launch of each feature kernel."""
        self._check(_lib.sttm_profile_enable(self._h, int(every)))

    def sttm_profile_read(self, kernel: int):
        ms, n = C.c_double(0.0), C.c_int64(0)
        self._check(_lib.sttm_profile_read(self._h, kernel, C.byref(ms), C.byref(n)))
        return float(ms.value), int(n.value)
