"""Thin ctypes binding of the C ABI in include/fvdb_hotpath.h.

Argument marshalling only: every step of the path runs inside the HIP library.  PyTorch is
used for device memory and for the current stream.  There is no CPU fallback: if the built
library is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Tuple

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfvdb_hotpath.so")

FX_OK = 0
DTYPES = {"f32": 0, "f16": 1, "bf16": 2}
_TORCH_DT = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
STATUS_NAMES = {0: "FX_OK", -1: "FX_EINVAL", -2: "FX_EUNSUPPORTED", -3: "FX_ENOMEM", -4: "FX_EDEVICE",
                -5: "FX_ERANGE"}

LEAF_DTYPE = np.dtype([("offset", "<i8"), ("prefix", "<u8"), ("mask", "<u8", (8,)),
                       ("origin", "<i4", (3,)), ("batch", "<i4")])


class FxError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class _BlockJoin(C.Structure):
    """fx_block_join"""
    _fields_ = [("rows", C.c_int64), ("C", C.c_int32), ("dt", C.c_int32), ("vec_dt", C.c_int32), ("act", C.c_int32),
                ("d_y", C.c_void_p), ("d_gate", C.c_void_p), ("ld_y", C.c_int64), ("ld_gate", C.c_int64),
                ("d_post", C.c_void_p), ("d_scale", C.c_void_p), ("d_next", C.c_void_p), ("d_offset", C.c_void_p),
                ("seed", C.c_uint64), ("offset", C.c_uint64), ("p", C.c_double), ("eps", C.c_float)]


class _Attention(C.Structure):
    """fx_attention"""
    _fields_ = [("q_seqs", C.c_void_p), ("kv_seqs", C.c_void_p), ("dt", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("dim", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float), ("d_q", C.c_void_p), ("d_k", C.c_void_p), ("d_v", C.c_void_p),
                ("ld_q", C.c_int64), ("hs_q", C.c_int64), ("ld_k", C.c_int64), ("hs_k", C.c_int64), ("ld_v", C.c_int64), ("hs_v", C.c_int64)]


class _Cache(C.Structure):
    """fx_cache"""
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("d_k_exp", C.c_void_p), ("d_v_exp", C.c_void_p), ("d_table", C.c_void_p),
                ("ld_table", C.c_int64), ("table_cols", C.c_int32), ("pages", C.c_int32), ("page_rows", C.c_int32), ("store", C.c_int32),
                ("kv_heads", C.c_int32), ("dim", C.c_int32)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2407_01781_amd.build` "
            "(there is no fallback implementation)")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    L.fx_version.restype = C.c_char_p
    L.fx_last_error.restype = C.c_char_p
    L.fx_init.restype = C.c_int
    L.fx_build_index_grid.restype = C.c_int
    L.fx_build_index_grid.argtypes = [vp, i64, vp, i32, vp, C.POINTER(vp)]
    L.fx_build_index_grid_from_points.restype = C.c_int
    L.fx_build_index_grid_from_points.argtypes = [vp, i64, vp, i32, vp, vp, vp, C.POINTER(vp)]
    L.fx_grid_info.restype = C.c_int
    L.fx_grid_info.argtypes = [vp, C.POINTER(i64), C.POINTER(i32), vp, vp]
    L.fx_grid_ijk.restype = C.c_int
    L.fx_grid_ijk.argtypes = [vp, vp, vp, vp]
    L.fx_grid_ijk_to_index.restype = C.c_int
    L.fx_grid_ijk_to_index.argtypes = [vp, vp, vp, i64, vp, vp]
    L.fx_grid_leaf_table.restype = C.c_int
    L.fx_grid_leaf_table.argtypes = [vp, vp, C.c_size_t, vp]
    L.fx_grid_coarsen2.restype = C.c_int
    L.fx_grid_coarsen2.argtypes = [vp, vp, C.POINTER(vp)]
    L.fx_grid_retain.argtypes = [vp]
    L.fx_grid_destroy.argtypes = [vp]
    L.fx_build_kernel_map_onto.restype = C.c_int
    L.fx_build_kernel_map_onto.argtypes = [vp, vp, i32, vp, C.POINTER(vp)]
    L.fx_build_kernel_map.restype = C.c_int
    L.fx_build_kernel_map.argtypes = [vp, i32, i32, vp, C.POINTER(vp), C.POINTER(vp)]
    L.fx_kmap_info.restype = C.c_int
    L.fx_kmap_info.argtypes = [vp, C.POINTER(i64), C.POINTER(i32), C.POINTER(i64), vp]
    L.fx_kmap_dense.restype = C.c_int
    L.fx_kmap_dense.argtypes = [vp, vp, vp]
    L.fx_kmap_tile_stats.restype = C.c_int
    L.fx_kmap_tile_stats.argtypes = [vp, vp]
    L.fx_kmap_tiled_bytes.restype = C.c_int
    L.fx_kmap_tiled_bytes.argtypes = [vp, C.POINTER(i64)]
    L.fx_kmap_destroy.argtypes = [vp]
    L.fx_sparse_conv_fwd.restype = C.c_int
    L.fx_sparse_conv_fwd.argtypes = [vp, vp, C.c_int, vp, i32, i32, vp, C.c_int, vp]
    L.fx_sparse_conv_fwd_noalloc.restype = C.c_int
    L.fx_sparse_conv_fwd_noalloc.argtypes = [vp, vp, C.c_int, vp, i32, i32, vp, C.c_int, vp]
    L.fx_sparse_conv_bwd_data.restype = C.c_int
    L.fx_sparse_conv_bwd_data.argtypes = [vp, vp, C.c_int, vp, i32, i32, vp, C.c_int, vp]
    L.fx_sparse_conv_bwd_weight.restype = C.c_int
    L.fx_sparse_conv_bwd_weight.argtypes = [vp, vp, vp, C.c_int, i32, i32, vp, C.c_int, vp]
    L.fx_grid_subdivide2.restype = C.c_int
    L.fx_grid_subdivide2.argtypes = [vp, vp, C.POINTER(vp)]
    L.fx_grid_pad.restype = C.c_int
    L.fx_grid_pad.argtypes = [vp, C.c_int32, vp, C.POINTER(vp)]
    L.fx_sparse_conv_leaf_fwd.restype = C.c_int
    L.fx_sparse_conv_leaf_fwd.argtypes = [vp, vp, C.c_int, vp, i32, i32, vp, C.c_int, vp]
    L.fx_sparse_conv_leaf_bwd_weight.restype = C.c_int
    L.fx_sparse_conv_leaf_bwd_weight.argtypes = [vp, vp, vp, C.c_int, i32, i32, vp, C.c_int, vp]
    L.fx_sparse_conv_leaf_bwd_data.restype = C.c_int
    L.fx_sparse_conv_leaf_bwd_data.argtypes = [vp, vp, C.c_int, vp, i32, i32, vp, C.c_int, vp]
    L.fx_sparse_conv_transpose_fwd.restype = C.c_int
    L.fx_sparse_conv_transpose_fwd.argtypes = [vp, vp, C.c_int, vp, i32, i32, vp, C.c_int, vp]
    L.fx_pool2.restype = C.c_int
    L.fx_pool2.argtypes = [vp, i32, vp, C.c_int, i32, vp, vp]
    L.fx_pool2_bwd.restype = C.c_int
    L.fx_pool2_bwd.argtypes = [vp, C.c_int, vp, vp, C.c_int, i32, vp, vp]
    L.fx_upsample2_bwd.restype = C.c_int
    L.fx_upsample2_bwd.argtypes = [vp, vp, C.c_int, i32, vp, vp]
    L.fx_upsample2.restype = C.c_int
    L.fx_upsample2.argtypes = [vp, vp, C.c_int, i32, vp, vp]
    f32, f64, u64 = C.c_float, C.c_double, C.c_uint64
    for name, args in (
            ("fx_build_sequences", [vp, i32, i64, vp, C.POINTER(vp)]),
            ("fx_gated_scan_fwd", [vp, vp, i64, vp, i64, C.c_int, i32, i32, vp, vp, i64, vp, vp]),
            ("fx_gated_scan_bwd", [vp, vp, i64, vp, i64, vp, i64, vp, i64, C.c_int, i32, i32, vp, vp, vp, i64, vp, i64, vp, vp]),
            ("fx_gated_scan_step", [vp, i64, vp, i64, C.c_int, i64, i32, vp, vp, vp, i64, vp]),
            ("fx_rms_norm_fwd", [vp, i64, C.c_int, i64, i32, vp, C.c_int, f32, vp, i64, vp]),
            ("fx_rms_norm_bwd", [vp, i64, vp, i64, C.c_int, i64, i32, vp, C.c_int, f32, vp, i64, vp, vp]),
            ("fx_block_join_fwd", [C.POINTER(_BlockJoin), vp, i64, vp, i64, vp, i64, vp]),
            ("fx_block_join_bwd", [C.POINTER(_BlockJoin), vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp]),
            ("fx_attention_fwd", [C.POINTER(_Attention), vp, i64, i64, vp, vp]),
            ("fx_attention_bwd", [C.POINTER(_Attention), vp, i64, i64, vp, vp, i64, i64, vp, vp, i64, i64, vp, i64, i64, vp, i64, i64, vp]),
            ("fx_cache_write", [C.POINTER(_Cache), vp, i64, vp, C.c_int, vp, i64, i64, vp, i64, i64, vp]),
            ("fx_cache_read", [C.POINTER(_Cache), vp, vp, C.c_int, vp, i64, i64, vp, i64, i64, vp]),
            ("fx_attention_step", [C.POINTER(_Cache), i64, vp, i64, C.c_int, i32, f32, vp, i64, i64, vp, i64, i64, vp, vp]),
            ("fx_dropout", [vp, i64, C.c_int, i64, i32, f64, u64, u64, vp, vp, i64, vp, i64, vp])):
        getattr(L, name).restype = C.c_int
        getattr(L, name).argtypes = args
    L.fx_sequences_destroy.restype = None
    L.fx_sequences_destroy.argtypes = [vp]
    L.fx_set_option.restype = C.c_int
    L.fx_set_option.argtypes = [C.c_char_p, i32]
    L.fx_get_option.restype = C.c_int
    L.fx_get_option.argtypes = [C.c_char_p, C.POINTER(i32)]
    L.fx_set_allocator.restype = C.c_int
    L.fx_set_allocator.argtypes = [vp, vp, vp]
    L.fx_release_cached_memory.restype = None
    L.fx_profile_enable.argtypes = [C.c_int]
    L.fx_profile_slot_count.restype = C.c_int
    L.fx_profile_slot_name.restype = C.c_char_p
    L.fx_profile_slot_name.argtypes = [C.c_int]
    L.fx_profile_read.restype = C.c_int
    L.fx_profile_read.argtypes = [C.c_int, C.POINTER(C.c_double), C.POINTER(i64)]
    return L


lib = _load()


def _check(status: int):
    if status != FX_OK:
        raise FxError(status, lib.fx_last_error().decode())


# the current stream's handle without the Stream object around it (2.8 us a call, of some 10 for a small operator)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def set_option(name: str, value: int) -> None:
    """Process-wide switch of the library (fx_set_option); -1 restores the automatic choice."""
    _check(lib.fx_set_option(name.encode(), int(value)))


def get_option(name: str) -> int:
    v = C.c_int32()
    _check(lib.fx_get_option(name.encode(), C.byref(v)))
    return v.value


_ALLOC_CB = C.CFUNCTYPE(C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p)
_FREE_CB = C.CFUNCTYPE(None, C.c_void_p, C.c_void_p, C.c_void_p)
_torch_alloc_cbs = None          # the callback objects must outlive their use by the library


def use_torch_allocator(enable: bool = True) -> None:
    """Let PyTorch's caching allocator back all device memory the library needs (fx_set_allocator), or go back
    to the library's own block cache.  Switch while no grid or kernel-map handle is alive."""
    global _torch_alloc_cbs
    if not enable:
        _check(lib.fx_set_allocator(None, None, None))
        _torch_alloc_cbs = None
        return

    def _alloc(nbytes, stream, _ctx):
        try:
            return torch.cuda.caching_allocator_alloc(int(nbytes), stream=int(stream or 0))
        except Exception:          # out of memory: the library reports FX_ENOMEM
            return None

    def _free(ptr, _stream, _ctx):
        torch.cuda.caching_allocator_delete(int(ptr))

    cbs = (_ALLOC_CB(_alloc), _FREE_CB(_free))
    _check(lib.fx_set_allocator(C.cast(cbs[0], C.c_void_p), C.cast(cbs[1], C.c_void_p), None))
    _torch_alloc_cbs = cbs


def version() -> str:
    return lib.fx_version().decode()


def profile_enable(on: bool) -> None:
    lib.fx_profile_enable(1 if on else 0)


def profile_reset() -> None:
    lib.fx_profile_reset()


def profile_read() -> dict:
    """{kernel slot name: (total ms, launches)} for slots with at least one launch."""
    out = {}
    for slot in range(lib.fx_profile_slot_count()):
        ms, cnt = C.c_double(), C.c_int64()
        _check(lib.fx_profile_read(slot, C.byref(ms), C.byref(cnt)))
        if cnt.value:
            out[lib.fx_profile_slot_name(slot).decode()] = (float(ms.value), int(cnt.value))
    return out


class IndexGrid:
    """Handle on a GridBatch built by fx_build_index_grid (or a coarsened / output grid)."""

    def __init__(self, handle: int):
        self._h = C.c_void_p(handle)
        n, b = C.c_int64(), C.c_int32()
        _check(lib.fx_grid_info(self._h, C.byref(n), C.byref(b), None, None))
        self.num_voxels, self.batch_size = int(n.value), int(b.value)

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            lib.fx_grid_destroy(h)
            self._h = None

    def counts(self) -> Tuple[int, int, int]:
        c = np.zeros(3, dtype=np.int64)
        _check(lib.fx_grid_info(self._h, None, None, None, c.ctypes.data_as(C.c_void_p)))
        return int(c[0]), int(c[1]), int(c[2])

    def voxel_joffsets(self) -> np.ndarray:
        out = np.zeros((self.batch_size, 2), dtype=np.int64)
        _check(lib.fx_grid_info(self._h, None, None, out.ctypes.data_as(C.c_void_p), None))
        return out

    def ijk(self) -> Tuple[torch.Tensor, torch.Tensor]:
        out = torch.empty((self.num_voxels, 3), dtype=torch.int32, device="cuda")
        jidx = torch.empty((self.num_voxels,), dtype=torch.int32, device="cuda")
        _check(lib.fx_grid_ijk(self._h, _ptr(out), _ptr(jidx), _stream()))
        return out, jidx

    def ijk_to_index(self, ijk: torch.Tensor, jidx: Optional[torch.Tensor] = None) -> torch.Tensor:
        assert ijk.is_cuda and ijk.dtype == torch.int32 and ijk.is_contiguous()
        n = ijk.shape[0]
        if jidx is not None:
            assert jidx.is_cuda and jidx.dtype == torch.int32 and jidx.is_contiguous() and jidx.shape[0] == n
        out = torch.empty((n,), dtype=torch.int32, device="cuda")
        _check(lib.fx_grid_ijk_to_index(self._h, _ptr(ijk), _ptr(jidx), n, _ptr(out), _stream()))
        return out

    def leaf_table(self) -> np.ndarray:
        n_leaf = self.counts()[0]
        out = np.zeros(n_leaf, dtype=LEAF_DTYPE)
        _check(lib.fx_grid_leaf_table(self._h, out.ctypes.data_as(C.c_void_p), out.nbytes, _stream()))
        return out

    def coarsen2(self) -> "IndexGrid":
        h = C.c_void_p()
        _check(lib.fx_grid_coarsen2(self._h, _stream(), C.byref(h)))
        return IndexGrid(h.value)

    def subdivide2(self) -> "IndexGrid":
        """The grid of all eight children of every voxel."""
        h = C.c_void_p()
        _check(lib.fx_grid_subdivide2(self._h, _stream(), C.byref(h)))
        return IndexGrid(h.value)

    def pad(self, r: int = 1) -> "IndexGrid":
        """The grid of all voxels within Chebyshev distance r of an active one."""
        h = C.c_void_p()
        _check(lib.fx_grid_pad(self._h, int(r), _stream(), C.byref(h)))
        return IndexGrid(h.value)


def build_index_grid(ijk: torch.Tensor, joffsets) -> IndexGrid:
    """ijk: CUDA int32 [n_rows,3]; joffsets: host int64 [B,2]."""
    assert ijk.is_cuda and ijk.dtype == torch.int32 and ijk.is_contiguous()
    jo = np.ascontiguousarray(np.asarray(joffsets, dtype=np.int64).reshape(-1, 2))
    h = C.c_void_p()
    _check(lib.fx_build_index_grid(_ptr(ijk), ijk.shape[0], jo.ctypes.data_as(C.c_void_p), jo.shape[0],
                                   _stream(), C.byref(h)))
    return IndexGrid(h.value)


def build_index_grid_from_points(xyz: torch.Tensor, joffsets, origin=(0.0, 0.0, 0.0),
                                 voxel_size=(1.0, 1.0, 1.0)) -> IndexGrid:
    """xyz: CUDA float32 [n_rows,3]; voxel (i,j,k) is the cell [origin + i*s, origin + (i+1)*s)."""
    assert xyz.is_cuda and xyz.dtype == torch.float32 and xyz.is_contiguous()
    jo = np.ascontiguousarray(np.asarray(joffsets, dtype=np.int64).reshape(-1, 2))
    o = np.ascontiguousarray(np.broadcast_to(np.asarray(origin, dtype=np.float32), (3,)))
    s = np.ascontiguousarray(np.broadcast_to(np.asarray(voxel_size, dtype=np.float32), (3,)))
    h = C.c_void_p()
    _check(lib.fx_build_index_grid_from_points(_ptr(xyz), xyz.shape[0], jo.ctypes.data_as(C.c_void_p), jo.shape[0],
                                               o.ctypes.data_as(C.c_void_p), s.ctypes.data_as(C.c_void_p),
                                               _stream(), C.byref(h)))
    return IndexGrid(h.value)


class KernelMap:
    def __init__(self, handle: int, g_in: IndexGrid, g_out: IndexGrid, kernel_size: int, stride: int):
        self._h = C.c_void_p(handle)
        self.g_in, self.g_out = g_in, g_out
        self.kernel_size, self.stride = kernel_size, stride
        self.k3 = kernel_size ** 3
        self.n_out = g_out.num_voxels

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            lib.fx_kmap_destroy(h)
            self._h = None

    def info(self) -> Tuple[int, np.ndarray]:
        """(number of active pairs, pairs per offset [K^3])."""
        n_out, k3, n_pairs = C.c_int64(), C.c_int32(), C.c_int64()
        per = np.zeros(self.k3, dtype=np.int64)
        _check(lib.fx_kmap_info(self._h, C.byref(n_out), C.byref(k3), C.byref(n_pairs),
                                per.ctypes.data_as(C.c_void_p)))
        return int(n_pairs.value), per

    def tile_stats(self) -> dict:
        s = np.zeros(4, dtype=np.int64)
        _check(lib.fx_kmap_tile_stats(self._h, s.ctypes.data_as(C.c_void_p)))
        return {"mfma_rows_issued": int(s[0]), "n_tiles": int(s[1]), "staged_rows": int(s[2]), "tile": int(s[3])}

    def tiled_bytes(self) -> int:
        b = C.c_int64()
        _check(lib.fx_kmap_tiled_bytes(self._h, C.byref(b)))
        return int(b.value)

    def dense(self) -> torch.Tensor:
        out = torch.empty((self.n_out, self.k3), dtype=torch.int32, device="cuda")
        _check(lib.fx_kmap_dense(self._h, _ptr(out), _stream()))
        return out


def release_cached_memory() -> None:
    """Return the device blocks the library keeps for reuse to the driver (waits for the device)."""
    lib.fx_release_cached_memory()


def build_kernel_map(g_in: IndexGrid, kernel_size: int, stride: int) -> KernelMap:
    hg, hk = C.c_void_p(), C.c_void_p()
    _check(lib.fx_build_kernel_map(g_in._h, kernel_size, stride, _stream(), C.byref(hg), C.byref(hk)))
    g_out = IndexGrid(hg.value)
    return KernelMap(hk.value, g_in, g_out, kernel_size, stride)


def build_kernel_map_onto(g_in: IndexGrid, g_out: IndexGrid, kernel_size: int) -> KernelMap:
    """Stride-1 map from the voxels of g_out (any grid of the same batch size) into g_in."""
    hk = C.c_void_p()
    _check(lib.fx_build_kernel_map_onto(g_in._h, g_out._h, kernel_size, _stream(), C.byref(hk)))
    return KernelMap(hk.value, g_in, g_out, kernel_size, 1)


def sparse_conv_fwd(kmap: KernelMap, feat: torch.Tensor, weights: torch.Tensor,
                    out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """feat [N_in, C_in], weights [K^3, C_in, C_out] (same dtype, CUDA, contiguous)."""
    assert feat.is_cuda and weights.is_cuda and feat.is_contiguous() and weights.is_contiguous()
    assert feat.dtype == weights.dtype and feat.dtype in _TORCH_DT
    k3, c_in, c_out = weights.shape
    assert k3 == kmap.k3 and feat.shape == (kmap.g_in.num_voxels, c_in)
    out_dtype = out_dtype or feat.dtype
    if out is None:
        out = torch.empty((kmap.n_out, c_out), dtype=out_dtype, device="cuda")
    assert out.is_cuda and out.is_contiguous() and out.shape == (kmap.n_out, c_out) and out.dtype == out_dtype
    _check(lib.fx_sparse_conv_fwd(kmap._h, _ptr(feat), _TORCH_DT[feat.dtype], _ptr(weights), c_in, c_out,
                                  _ptr(out), _TORCH_DT[out_dtype], _stream()))
    return out


def sparse_conv_fwd_noalloc(kmap: KernelMap, feat: torch.Tensor, weights: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """sparse_conv_fwd through the entry point that allocates nothing; the caller supplies `out` [N_out, C_out]."""
    assert feat.is_cuda and weights.is_cuda and feat.is_contiguous() and weights.is_contiguous()
    assert feat.dtype == weights.dtype and feat.dtype in _TORCH_DT
    k3, c_in, c_out = weights.shape
    assert k3 == kmap.k3 and feat.shape == (kmap.g_in.num_voxels, c_in)
    assert out.is_cuda and out.is_contiguous() and out.shape == (kmap.n_out, c_out) and out.dtype in _TORCH_DT
    _check(lib.fx_sparse_conv_fwd_noalloc(kmap._h, _ptr(feat), _TORCH_DT[feat.dtype], _ptr(weights), c_in, c_out,
                                          _ptr(out), _TORCH_DT[out.dtype], _stream()))
    return out


def sparse_conv_bwd_data(kmap: KernelMap, grad_out: torch.Tensor, weights: torch.Tensor,
                         out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """grad_out [N_out, C_out], weights [K^3, C_in, C_out] -> gradient of the input features [N_in, C_in]."""
    assert grad_out.is_cuda and weights.is_cuda and grad_out.is_contiguous() and weights.is_contiguous()
    assert grad_out.dtype == weights.dtype and grad_out.dtype in _TORCH_DT
    k3, c_in, c_out = weights.shape
    assert k3 == kmap.k3 and grad_out.shape == (kmap.n_out, c_out)
    out_dtype = out_dtype or grad_out.dtype
    gin = out if out is not None else torch.empty((kmap.g_in.num_voxels, c_in), dtype=out_dtype, device="cuda")
    assert gin.is_cuda and gin.is_contiguous() and gin.shape == (kmap.g_in.num_voxels, c_in) and gin.dtype == out_dtype
    _check(lib.fx_sparse_conv_bwd_data(kmap._h, _ptr(grad_out), _TORCH_DT[grad_out.dtype], _ptr(weights), c_in, c_out,
                                       _ptr(gin), _TORCH_DT[out_dtype], _stream()))
    return gin


def sparse_conv_bwd_weight(kmap: KernelMap, feat: torch.Tensor, grad_out: torch.Tensor,
                           out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """feat [N_in, C_in], grad_out [N_out, C_out] -> gradient of the weights [K^3, C_in, C_out]."""
    assert feat.is_cuda and grad_out.is_cuda and feat.is_contiguous() and grad_out.is_contiguous()
    assert feat.dtype == grad_out.dtype and feat.dtype in _TORCH_DT
    c_in, c_out = feat.shape[1], grad_out.shape[1]
    assert feat.shape[0] == kmap.g_in.num_voxels and grad_out.shape[0] == kmap.n_out
    out_dtype = out_dtype or feat.dtype
    gw = out if out is not None else torch.empty((kmap.k3, c_in, c_out), dtype=out_dtype, device="cuda")
    assert gw.is_cuda and gw.is_contiguous() and gw.shape == (kmap.k3, c_in, c_out) and gw.dtype == out_dtype
    _check(lib.fx_sparse_conv_bwd_weight(kmap._h, _ptr(feat), _ptr(grad_out), _TORCH_DT[feat.dtype], c_in, c_out,
                                         _ptr(gw), _TORCH_DT[out_dtype], _stream()))
    return gw


def sparse_conv_transpose_fwd(kmap: KernelMap, feat: torch.Tensor, weights: torch.Tensor,
                              out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """feat [N_out, C_in] on the map's output grid, weights [K^3, C_in, C_out] -> [N_in, C_out] on its input grid."""
    assert feat.is_cuda and weights.is_cuda and feat.is_contiguous() and weights.is_contiguous()
    assert feat.dtype == weights.dtype and feat.dtype in _TORCH_DT
    k3, c_in, c_out = weights.shape
    assert k3 == kmap.k3 and feat.shape == (kmap.n_out, c_in)
    out_dtype = out_dtype or feat.dtype
    out = torch.empty((kmap.g_in.num_voxels, c_out), dtype=out_dtype, device="cuda")
    _check(lib.fx_sparse_conv_transpose_fwd(kmap._h, _ptr(feat), _TORCH_DT[feat.dtype], _ptr(weights), c_in, c_out,
                                            _ptr(out), _TORCH_DT[out_dtype], _stream()))
    return out


def sparse_conv_leaf_fwd(grid: IndexGrid, feat: torch.Tensor, weights: torch.Tensor,
                         out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """3x3x3 submanifold convolution straight from the grid (no kernel map): feat [N, C_in],
    weights [27, C_in, C_out] -> [N, C_out]; fp32 at low depth, f16 / bf16 at C_in % 32 == 0, C_out % 64 == 0."""
    assert feat.is_cuda and weights.is_cuda and feat.is_contiguous() and weights.is_contiguous()
    assert feat.dtype == weights.dtype and feat.dtype in _TORCH_DT
    k3, c_in, c_out = weights.shape
    assert k3 == 27 and feat.shape == (grid.num_voxels, c_in)
    out_dtype = out_dtype or feat.dtype
    out = torch.empty((grid.num_voxels, c_out), dtype=out_dtype, device="cuda")
    _check(lib.fx_sparse_conv_leaf_fwd(grid._h, _ptr(feat), _TORCH_DT[feat.dtype], _ptr(weights), c_in, c_out,
                                       _ptr(out), _TORCH_DT[out_dtype], _stream()))
    return out


def sparse_conv_leaf_bwd_data(grid: IndexGrid, grad_out: torch.Tensor, weights: torch.Tensor,
                              out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """Input gradient of sparse_conv_leaf_fwd: grad_out [N, C_out], weights [27, C_in, C_out] -> [N, C_in]."""
    assert grad_out.is_cuda and weights.is_cuda and grad_out.is_contiguous() and weights.is_contiguous()
    assert grad_out.dtype == weights.dtype and grad_out.dtype in _TORCH_DT
    k3, c_in, c_out = weights.shape
    assert k3 == 27 and grad_out.shape == (grid.num_voxels, c_out)
    out_dtype = out_dtype or grad_out.dtype
    gin = torch.empty((grid.num_voxels, c_in), dtype=out_dtype, device="cuda")
    _check(lib.fx_sparse_conv_leaf_bwd_data(grid._h, _ptr(grad_out), _TORCH_DT[grad_out.dtype], _ptr(weights), c_in, c_out,
                                            _ptr(gin), _TORCH_DT[out_dtype], _stream()))
    return gin


def sparse_conv_leaf_bwd_weight(grid: IndexGrid, feat: torch.Tensor, grad_out: torch.Tensor,
                                out_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """Weight gradient of sparse_conv_leaf_fwd: feat [N, C_in], grad_out [N, C_out] -> [27, C_in, C_out]."""
    assert feat.is_cuda and grad_out.is_cuda and feat.is_contiguous() and grad_out.is_contiguous()
    assert feat.dtype == grad_out.dtype and feat.dtype in _TORCH_DT
    assert feat.shape[0] == grid.num_voxels and grad_out.shape[0] == grid.num_voxels
    c_in, c_out = feat.shape[1], grad_out.shape[1]
    out_dtype = out_dtype or feat.dtype
    gw = torch.empty((27, c_in, c_out), dtype=out_dtype, device="cuda")
    _check(lib.fx_sparse_conv_leaf_bwd_weight(grid._h, _ptr(feat), _ptr(grad_out), _TORCH_DT[feat.dtype], c_in, c_out,
                                              _ptr(gw), _TORCH_DT[out_dtype], _stream()))
    return gw


def pool2(kmap: KernelMap, feat: torch.Tensor, mode: str = "max") -> torch.Tensor:
    """Max / mean over the active children; kmap is a (2,2) map, feat [N_in, C] -> [N_out, C]."""
    assert feat.is_cuda and feat.is_contiguous() and feat.dtype in _TORCH_DT
    assert feat.shape[0] == kmap.g_in.num_voxels
    out = torch.empty((kmap.n_out, feat.shape[1]), dtype=feat.dtype, device="cuda")
    _check(lib.fx_pool2(kmap._h, {"max": 0, "avg": 1}[mode], _ptr(feat), _TORCH_DT[feat.dtype], feat.shape[1],
                        _ptr(out), _stream()))
    return out


def upsample2(kmap: KernelMap, feat: torch.Tensor) -> torch.Tensor:
    """Nearest-neighbour upsampling; kmap is a (2,2) map, feat [N_out, C] -> [N_in, C]."""
    assert feat.is_cuda and feat.is_contiguous() and feat.dtype in _TORCH_DT
    assert feat.shape[0] == kmap.n_out
    out = torch.empty((kmap.g_in.num_voxels, feat.shape[1]), dtype=feat.dtype, device="cuda")
    _check(lib.fx_upsample2(kmap._h, _ptr(feat), _TORCH_DT[feat.dtype], feat.shape[1], _ptr(out), _stream()))
    return out


def pool2_bwd(kmap: KernelMap, grad_out: torch.Tensor, mode: str = "max", feat: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of pool2: grad_out [N_out, C] -> [N_in, C]; max pooling needs the forward input feat [N_in, C]."""
    assert grad_out.is_cuda and grad_out.is_contiguous() and grad_out.dtype in _TORCH_DT and grad_out.shape[0] == kmap.n_out
    if mode == "max":
        assert feat is not None and feat.is_cuda and feat.is_contiguous() and feat.dtype == grad_out.dtype
        assert feat.shape == (kmap.g_in.num_voxels, grad_out.shape[1])
    gin = torch.empty((kmap.g_in.num_voxels, grad_out.shape[1]), dtype=grad_out.dtype, device="cuda")
    _check(lib.fx_pool2_bwd(kmap._h, {"max": 0, "avg": 1}[mode], _ptr(feat) if mode == "max" else None, _ptr(grad_out),
                            _TORCH_DT[grad_out.dtype], grad_out.shape[1], _ptr(gin), _stream()))
    return gin


def upsample2_bwd(kmap: KernelMap, grad_out: torch.Tensor) -> torch.Tensor:
    """Gradient of upsample2: grad_out [N_in, C] on the fine grid -> [N_out, C], the sum over the children."""
    assert grad_out.is_cuda and grad_out.is_contiguous() and grad_out.dtype in _TORCH_DT
    assert grad_out.shape[0] == kmap.g_in.num_voxels
    gin = torch.empty((kmap.n_out, grad_out.shape[1]), dtype=grad_out.dtype, device="cuda")
    _check(lib.fx_upsample2_bwd(kmap._h, _ptr(grad_out), _TORCH_DT[grad_out.dtype], grad_out.shape[1], _ptr(gin), _stream()))
    return gin


# ------------------------------------------------------------------------------------------ around the convolution
class Sequences:
    """Handle on the rows' division into sequences (fx_build_sequences).  Calls on any stream may use it; let go of it when
    those on other streams than the one it was built on have ended, and keep it for as long as a graph that uses it."""

    def __init__(self, handle: int, batch_size: int, rows: int):
        self._h = C.c_void_p(handle)
        self.batch_size, self.rows = batch_size, rows

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and lib is not None:        # None when the interpreter ends
            lib.fx_sequences_destroy(h)
            self._h = None


def build_sequences(joffsets) -> Sequences:
    """joffsets: host int64 [B,2], ranges that follow each other from row 0 on (IndexGrid.voxel_joffsets() makes every
    grid of a batch one sequence)."""
    jo = np.ascontiguousarray(np.asarray(joffsets, dtype=np.int64).reshape(-1, 2))
    rows = int(jo[-1, 1]) if len(jo) else 0
    h = C.c_void_p()
    _check(lib.fx_build_sequences(jo.ctypes.data_as(C.c_void_p), jo.shape[0], rows, _stream(), C.byref(h)))
    return Sequences(h.value, jo.shape[0], rows)


def _rows(t: torch.Tensor, like: torch.Tensor, name: str) -> int:
    """The address of a tensor of rows, of the shape and dtype of `like`: any row stride, channels next to each other."""
    if t.dtype != like.dtype or t.shape != like.shape or not t.is_cuda:
        raise AssertionError(f"{name}: {tuple(like.shape)} {like.dtype} on the GPU expected")
    if t.stride(1) != 1 and t.shape[1] > 1 and t.numel():
        raise AssertionError(f"{name}: the channels of a row have to lie next to each other")
    return t.data_ptr()


def _opt_rows(t: Optional[torch.Tensor], like: torch.Tensor, name: str):
    return None if t is None else _rows(t, like, name)


def _ld(t: Optional[torch.Tensor]) -> int:
    # the stride of a single row says nothing; rows of a broadcast tensor (stride 0) are refused by the library
    if t is None:
        return 0
    return t.stride(0) if t.shape[0] > 1 and t.shape[1] else max(t.shape[1], 1)


def _new_rows(like: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(like, memory_format=torch.contiguous_format)


def _out_rows(out: Optional[torch.Tensor], like: torch.Tensor) -> torch.Tensor:
    if out is None:
        return _new_rows(like)
    _rows(out, like, "out")
    return out


def _states(t: Optional[torch.Tensor], shape, name: str):
    if t is None:
        return None
    assert t.is_cuda and t.dtype == torch.float32 and t.shape == shape and t.is_contiguous(), \
        f"{name}: contiguous float32 {tuple(shape)} on the GPU expected"
    return t.data_ptr()


def _vector(t: Optional[torch.Tensor], like: torch.Tensor, name: str):
    if t is None:
        return None
    assert t.is_cuda and t.shape == like.shape[1:] and t.is_contiguous() and t.dtype in (like.dtype, torch.float32), \
        f"{name}: contiguous ({like.shape[1]},) of {like.dtype} or float32 on the GPU expected"
    return t.data_ptr()


def gated_scan_fwd(seqs: Sequences, x: torch.Tensor, gate: torch.Tensor, h0: Optional[torch.Tensor] = None, reverse: bool = False,
                   out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """h_t = f_t h_(t-1) + (1 - f_t) x_t with f = sigmoid(gate) along every sequence, against the rows' order where
    `reverse`; x, gate [rows, C], h0 [B, C] float32 (zeros without).  Returns h [rows, C] and the states [B, C] float32
    behind the last rows."""
    assert x.dim() == 2 and x.dtype in _TORCH_DT and x.shape[0] == seqs.rows
    xp, gp = _rows(x, x, "x"), _rows(gate, x, "gate")
    states = (seqs.batch_size, x.shape[1])
    h0p = _states(h0, states, "h0")
    h = _out_rows(out, x)
    last = torch.empty(states, dtype=torch.float32, device=x.device)
    _check(lib.fx_gated_scan_fwd(seqs._h, xp, _ld(x), gp, _ld(gate), _TORCH_DT[x.dtype], x.shape[1], int(reverse), h0p, h.data_ptr(),
                                 _ld(h), last.data_ptr(), _stream()))
    return h, last


def gated_scan_bwd(seqs: Sequences, x: torch.Tensor, gate: torch.Tensor, h: torch.Tensor, grad_h: torch.Tensor,
                   h0: Optional[torch.Tensor] = None, grad_last: Optional[torch.Tensor] = None,
                   reverse: bool = False) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients of gated_scan_fwd's x, gate [rows, C] and h0 [B, C]; h is its output, grad_last the gradient of its
    second output (zeros without)."""
    assert x.dim() == 2 and x.dtype in _TORCH_DT and x.shape[0] == seqs.rows
    xp, gp, hp, ghp = _rows(x, x, "x"), _rows(gate, x, "gate"), _rows(h, x, "h"), _rows(grad_h, x, "grad_h")
    states = (seqs.batch_size, x.shape[1])
    h0p, glp = _states(h0, states, "h0"), _states(grad_last, states, "grad_last")
    gx, ggate = _new_rows(x), _new_rows(x)
    gh0 = torch.empty(states, dtype=torch.float32, device=x.device)
    _check(lib.fx_gated_scan_bwd(seqs._h, xp, _ld(x), gp, _ld(gate), hp, _ld(h), ghp, _ld(grad_h), _TORCH_DT[x.dtype], x.shape[1],
                                 int(reverse), h0p, glp, gx.data_ptr(), _ld(gx), ggate.data_ptr(), _ld(ggate), gh0.data_ptr(), _stream()))
    return gx, ggate, gh0


def gated_scan_step(x: torch.Tensor, gate: torch.Tensor, state: torch.Tensor,
                    new_state: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The next row of each of x.shape[0] running sequences: h [n, C] and the states behind it [n, C] float32
    (new_state may be `state`)."""
    assert x.dim() == 2 and x.dtype in _TORCH_DT
    xp, gp = _rows(x, x, "x"), _rows(gate, x, "gate")
    sp = _states(state, x.shape, "state")
    h = _new_rows(x)
    if new_state is None:
        new_state = torch.empty_like(state)
    _check(lib.fx_gated_scan_step(xp, _ld(x), gp, _ld(gate), _TORCH_DT[x.dtype], x.shape[0], x.shape[1], sp,
                                  _states(new_state, x.shape, "new_state"), h.data_ptr(), _ld(h), _stream()))
    return h, new_state


def rms_norm_fwd(x: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x / sqrt(mean over the channels of x^2 + eps) * weight; x [rows, C], weight [C] of x's dtype or float32."""
    assert x.dim() == 2 and x.dtype in _TORCH_DT
    xp, wp = _rows(x, x, "x"), _vector(weight, x, "weight")
    out = _out_rows(out, x)
    _check(lib.fx_rms_norm_fwd(xp, _ld(x), _TORCH_DT[x.dtype], x.shape[0], x.shape[1], wp, 0 if weight is None else _TORCH_DT[weight.dtype],
                               eps, out.data_ptr(), _ld(out), _stream()))
    return out


def rms_norm_bwd(grad_out: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor] = None,
                 eps: float = 1e-6) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Gradients of rms_norm_fwd's x and weight (None without one)."""
    assert x.dim() == 2 and x.dtype in _TORCH_DT
    xp, gp, wp = _rows(x, x, "x"), _rows(grad_out, x, "grad_out"), _vector(weight, x, "weight")
    gx = _new_rows(x)
    gw = None if weight is None else torch.empty_like(weight)
    _check(lib.fx_rms_norm_bwd(gp, _ld(grad_out), xp, _ld(x), _TORCH_DT[x.dtype], x.shape[0], x.shape[1], wp,
                               0 if weight is None else _TORCH_DT[weight.dtype], eps, gx.data_ptr(), _ld(gx),
                               None if gw is None else gw.data_ptr(), _stream()))
    return gx, gw


_GATES = {"sigmoid": 0, "silu": 1}


def _offset(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.dtype == torch.int64 and t.numel() == 1, "d_offset: one int64 on the GPU"
    return t.data_ptr()


def _block(y, gate, act, post_weight, scale, next_weight, eps, p, seed, offset, d_offset) -> _BlockJoin:
    assert y.dim() == 2 and y.dtype in _TORCH_DT
    some = post_weight if post_weight is not None else scale if scale is not None else next_weight
    vec = torch.float32 if some is None else some.dtype
    assert all(v is None or v.dtype == vec for v in (scale, next_weight)), "post_weight, scale and next_weight have one dtype"
    # in the order of the members
    return _BlockJoin(y.shape[0], y.shape[1], _TORCH_DT[y.dtype], _TORCH_DT[vec], _GATES[act], _rows(y, y, "y"),
                      _opt_rows(gate, y, "gate"), _ld(y), _ld(gate), _vector(post_weight, y, "post_weight"), _vector(scale, y, "scale"),
                      _vector(next_weight, y, "next_weight"), _offset(d_offset), seed, offset, p, eps)


def block_join_fwd(x: torch.Tensor, y: torch.Tensor, gate: Optional[torch.Tensor] = None, act: str = "silu",
                   post_weight: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                   next_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, p: float = 0.0, seed: int = 0, offset: int = 0,
                   d_offset: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """x + scale * drop(rms_norm(y; post_weight) * act(gate)), and that sum's rms_norm by next_weight (None without one).
    Rows [n, C] of one dtype, vectors [C] of that dtype or float32; drop is dropout's mask of (seed, offset)."""
    b = _block(y, gate, act, post_weight, scale, next_weight, eps, p, seed, offset, d_offset)
    xp = _rows(x, y, "x")
    out = _out_rows(out, x)
    norm = None if next_weight is None else _new_rows(x)
    _check(lib.fx_block_join_fwd(b, xp, _ld(x), out.data_ptr(), _ld(out), None if norm is None else norm.data_ptr(), _ld(norm), _stream()))
    return out, norm


def block_join_bwd(grad_out: Optional[torch.Tensor], grad_norm: Optional[torch.Tensor], out: Optional[torch.Tensor], y: torch.Tensor,
                   gate: Optional[torch.Tensor] = None, act: str = "silu", post_weight: Optional[torch.Tensor] = None,
                   scale: Optional[torch.Tensor] = None, next_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, p: float = 0.0,
                   seed: int = 0, offset: int = 0, d_offset: Optional[torch.Tensor] = None) -> dict:
    """Gradients of block_join_fwd's inputs: {"x", "y", "gate", "post", "scale", "next"}, None for those that are absent.
    grad_out and grad_norm are the gradients of its two outputs (one may be None), `out` its first output (needed with
    grad_norm)."""
    b = _block(y, gate, act, post_weight, scale, next_weight, eps, p, seed, offset, d_offset)
    ins = []
    for t, name in ((grad_out, "grad_out"), (grad_norm, "grad_norm"), (out, "out")):
        ins += (_opt_rows(t, y, name), _ld(t))
    rows = lambda t: None if t is None else _new_rows(y)
    vec = lambda t: None if t is None else torch.empty_like(t)
    g = {"x": _new_rows(y), "y": _new_rows(y), "gate": rows(gate), "post": vec(post_weight), "scale": vec(scale), "next": vec(next_weight)}
    ptr = [None if t is None else t.data_ptr() for t in g.values()]
    ld = max(y.shape[1], 1)
    _check(lib.fx_block_join_bwd(b, *ins, ptr[0], ld, ptr[1], ld, ptr[2], ld, *ptr[3:], _stream()))
    return g


def dropout(x: torch.Tensor, p: float, seed: int, offset: int, residual: Optional[torch.Tensor] = None,
            d_offset: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows, C] with a share p of its values dropped and the others scaled by 1 / (1 - p), plus the residual if there
    is one.  The mask depends on (seed, offset, row, channel) alone and is never stored; the gradient of x is the same
    call on the output's gradient.  Take another offset for every call that wants a mask of its own."""
    assert x.dim() == 2 and x.dtype in _TORCH_DT
    xp, rp = _rows(x, x, "x"), _opt_rows(residual, x, "residual")
    out = _out_rows(out, x)
    _check(lib.fx_dropout(xp, _ld(x), _TORCH_DT[x.dtype], x.shape[0], x.shape[1], p, seed, offset, _offset(d_offset), rp, _ld(residual),
                          out.data_ptr(), _ld(out), _stream()))
    return out


# ------------------------------------------------------------------------------------------ attention
class _Broadcast(AssertionError):
    """Rows, heads or elements lie on each other, as in the gradient of a sum: inputs are copied then."""


def _heads(t: torch.Tensor, shape, dtype: torch.dtype, device: int, name: str):
    """Address and strides from row to row and head to head of a tensor of heads [rows, heads, dim]: any order of rows and
    heads, a head's elements next to each other."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        raise AssertionError(f"{name}: {tuple(shape)} {dtype} on the current GPU expected")
    ld, hs, one = t.stride()
    rows, heads, dim = shape
    if not (ld and hs and one == 1) and rows:
        if ld == 0 and rows > 1 or hs == 0 and heads > 1 or one == 0 and dim > 1:
            raise _Broadcast(f"{name}: rows, heads and elements have to lie apart")
        if one != 1 and dim > 1:
            raise AssertionError(f"{name}: a head's elements have to lie next to each other")
    # the stride of a single row or head says nothing
    if heads <= 1:
        hs = dim
    return t.data_ptr(), (ld if rows > 1 else max(hs, dim) * max(heads, 1)), hs


def _new_heads(like: torch.Tensor):
    """A tensor of heads in new memory, and its address and strides."""
    t = torch.empty_like(like, memory_format=torch.contiguous_format)
    _, heads, dim = like.shape
    return t, t.data_ptr(), max(heads, 1) * dim, dim


def _floats(t: Optional[torch.Tensor], shape, device: int, name: str):
    if t is None:
        return None
    assert t.get_device() == device and t.dtype is torch.float32 and t.shape == shape and t.is_contiguous(), \
        f"{name}: contiguous float32 {tuple(shape)} on the current GPU expected"
    return t.data_ptr()


def _numbers(t: torch.Tensor, n: int, device: int, name: str) -> int:
    assert t.get_device() == device and t.dtype is torch.int32 and t.shape == (n,) and t.is_contiguous(), f"{name}: contiguous int32 ({n},) on the current GPU expected"
    return t.data_ptr()


def _attention(seqs: Sequences, kv_seqs: Optional[Sequences], q, k, v, causal: bool, scale: Optional[float], device: int) -> _Attention:
    assert q.dim() == 3 and k.dim() == 3 and q.dtype in _TORCH_DT, "q, k, v: [rows, heads, dim]"
    rows, heads, dim = shape = q.shape
    dtype = q.dtype
    assert rows == seqs.rows, f"q: {seqs.rows} rows expected"
    kv = (seqs if kv_seqs is None else kv_seqs).rows, k.shape[1], dim
    # in the order of the members
    (qp, lq, hq), (kp, lk, hk), (vp, lv, hv) = _heads(q, shape, dtype, device, "q"), _heads(k, kv, dtype, device, "k"), _heads(v, kv, dtype, device, "v")
    return _Attention(seqs._h, None if kv_seqs is None else kv_seqs._h, _TORCH_DT[dtype], heads, kv[1], dim, causal,
                      dim ** -0.5 if scale is None else scale, qp, kp, vp, lq, hq, lk, hk, lv, hv)


def attention_fwd(seqs: Sequences, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False, scale: Optional[float] = None,
                  kv_seqs: Optional[Sequences] = None, out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Softmax attention of every row over the rows of its sequence: q [rows, heads, dim], k and v [rows, kv_heads, dim] (query
    head h reads key head h // (heads / kv_heads)), or rows of kv_seqs, as many sequences.  causal: the last query stands at the last
    key, and none sees a later one.  scale: dim ** -0.5 without.  A head's elements lie next to each other; inputs that are broadcast
    are copied first.  Returns out [rows, heads, dim] and lse [heads, rows] float32, the
    logarithm of the sum of exp(scale q . k); 0 and -inf for a row that sees no key."""
    device = torch.cuda.current_device()
    try:
        a = _attention(seqs, kv_seqs, q, k, v, causal, scale, device)
    except _Broadcast:
        return attention_fwd(seqs, q.contiguous(), k.contiguous(), v.contiguous(), causal, scale, kv_seqs, out)
    out, *op = _new_heads(q) if out is None else (out, *_heads(out, q.shape, q.dtype, device, "out"))
    lse = torch.empty((a.heads, seqs.rows), dtype=torch.float32, device=q.device)
    _check(lib.fx_attention_fwd(a, *op, lse.data_ptr(), _stream()))
    return out, lse


def attention_bwd(seqs: Sequences, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                  grad_out: torch.Tensor, grad_lse: Optional[torch.Tensor] = None, causal: bool = False, scale: Optional[float] = None,
                  kv_seqs: Optional[Sequences] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients of attention_fwd's q, k and v; out and lse are its outputs, grad_lse the gradient of the second (zeros without)."""
    device = torch.cuda.current_device()
    try:
        a = _attention(seqs, kv_seqs, q, k, v, causal, scale, device)
        op, gp = _heads(out, q.shape, q.dtype, device, "out"), _heads(grad_out, q.shape, q.dtype, device, "grad_out")
    except _Broadcast:
        return attention_bwd(seqs, *(t.contiguous() for t in (q, k, v, out)), lse, grad_out.contiguous(), grad_lse, causal, scale, kv_seqs)
    stats = (q.shape[1], q.shape[0])
    lp, glp = _floats(lse, stats, device, "lse"), _floats(grad_lse, stats, device, "grad_lse")
    (gq, *gqp), (gk, *gkp), (gv, *gvp) = _new_heads(q), _new_heads(k), _new_heads(v)
    _check(lib.fx_attention_bwd(a, *op, lp, *gp, glp, *gqp, *gkp, *gvp, _stream()))
    return gq, gk, gv


class KVCache:
    """Keys and values of running sequences in pages (fx_cache): k and v [pages, kv_heads, page_rows, dim rounded up to 16], float32,
    float16, bfloat16 or float8_e4m3fn; the last with exponents k_exp and v_exp [pages, kv_heads, page_rows] uint8 (a value is
    code * 2 ** (exponent - 127)).  Which page a position has is said by the table of a call, [sequences, columns] int32: position p is row
    p % page_rows of page table[b, p // page_rows]; -1, or any other number that is no page, for those that have none."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, dim: Optional[int] = None, k_exp: Optional[torch.Tensor] = None,
                 v_exp: Optional[torch.Tensor] = None):
        assert k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.is_contiguous() and v.is_contiguous() and k.is_cuda and v.is_cuda, \
            "k and v: contiguous [pages, kv_heads, page_rows, dim rounded up to 16] of one type on the GPU"
        self.dim = k.shape[3] if dim is None else dim
        assert -(-self.dim // 16) * 16 == k.shape[3], f"rows of {k.shape[3]} elements do not hold {self.dim} dimensions rounded up to 16"
        e4m3 = k.dtype == torch.float8_e4m3fn
        assert e4m3 or k.dtype in _TORCH_DT, "float32, float16, bfloat16 or float8_e4m3fn expected"
        for t in (k_exp, v_exp):
            assert (t is not None) == e4m3, "exponents belong to a cache of 8 bits"
            assert t is None or (t.is_cuda and t.dtype == torch.uint8 and t.shape == k.shape[:3] and t.is_contiguous()), "exponents: contiguous uint8 [pages, kv_heads, page_rows]"
        self.k, self.v, self.k_exp, self.v_exp = k, v, k_exp, v_exp
        self.kv_heads, self._device = k.shape[1], k.get_device()
        self._c = _Cache(k.data_ptr(), v.data_ptr(), None if k_exp is None else k_exp.data_ptr(), None if v_exp is None else v_exp.data_ptr(), None, 0, 0,
                         k.shape[0], k.shape[2], 3 if e4m3 else _TORCH_DT[k.dtype], k.shape[1], self.dim)

    @classmethod
    def empty(cls, pages: int, page_rows: int, kv_heads: int, dim: int, dtype: torch.dtype = torch.bfloat16) -> "KVCache":
        """A cache of zeros in new memory."""
        new = lambda: torch.zeros((pages, kv_heads, page_rows, -(-dim // 16) * 16), dtype=dtype, device="cuda")
        exp = lambda: torch.zeros((pages, kv_heads, page_rows), dtype=torch.uint8, device="cuda") if dtype == torch.float8_e4m3fn else None
        return cls(new(), new(), dim, exp(), exp())

    def _with(self, table: torch.Tensor, n: int, device: int) -> _Cache:
        assert table.dtype is torch.int32 and table.dim() == 2 and table.shape[0] == n and (table.stride(1) == 1 or table.shape[1] <= 1), \
            f"table: int32 [{n}, columns] expected"
        assert self._device == device and table.get_device() == device, "cache and table have to be on the current GPU"
        c, cols = _Cache.from_buffer_copy(self._c), table.shape[1]
        c.d_table, c.table_cols, c.ld_table = table.data_ptr(), cols, table.stride(0) if n > 1 else max(cols, 1)
        return c


def cache_write(cache: KVCache, table: torch.Tensor, start: torch.Tensor, k: torch.Tensor, v: torch.Tensor, seqs: Optional[Sequences] = None) -> None:
    """Row r of sequence b of k and v [rows, kv_heads, dim] becomes position start[b] + r of the cache, rounded to its type; without
    seqs row b is one new row of sequence b.  No two rows may have one place; those whose position has no page are left out."""
    n = k.shape[0] if seqs is None else seqs.batch_size
    rows = k.shape[0] if seqs is None else seqs.rows
    device = torch.cuda.current_device()
    c = cache._with(table, n, device)
    assert k.dtype in _TORCH_DT, "k and v: float32, float16 or bfloat16"
    shape = rows, cache.kv_heads, cache.dim
    try:
        kp, vp = _heads(k, shape, k.dtype, device, "k"), _heads(v, shape, k.dtype, device, "v")
    except _Broadcast:
        return cache_write(cache, table, start, k.contiguous(), v.contiguous(), seqs)
    _check(lib.fx_cache_write(c, None if seqs is None else seqs._h, rows, _numbers(start, n, device, "start"), _TORCH_DT[k.dtype], *kp, *vp, _stream()))


def cache_read(cache: KVCache, table: torch.Tensor, start: torch.Tensor, seqs: Sequences,
               dtype: Optional[torch.dtype] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Keys and values [rows, kv_heads, dim] at the positions from start[b] on of every sequence, one for each of its rows of seqs
    (zeros for those that have no page); dtype: the cache's, which has to be said for one of 8 bits."""
    dtype = cache.k.dtype if dtype is None else dtype
    assert dtype in _TORCH_DT, "dtype: float32, float16 or bfloat16"
    device = torch.cuda.current_device()
    c = cache._with(table, seqs.batch_size, device)
    shape = seqs.rows, cache.kv_heads, cache.dim
    k = torch.empty(shape, dtype=dtype, device=cache.k.device)
    v = torch.empty_like(k)
    ld, hs = max(shape[1] * shape[2], 1), shape[2]
    _check(lib.fx_cache_read(c, seqs._h, _numbers(start, seqs.batch_size, device, "start"), _TORCH_DT[dtype], k.data_ptr(), ld, hs, v.data_ptr(), ld, hs, _stream()))
    return k, v


def attention_step(cache: KVCache, table: torch.Tensor, lengths: torch.Tensor, q: torch.Tensor, scale: Optional[float] = None,
                   longest: int = 0, out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of one new row of each of q.shape[0] running sequences, q [n, heads, dim], over the first lengths[b] positions that
    the cache holds of it.  longest: what no length passes (longer ones are cut there), if the program knows better than the table's width.  Returns out [n, heads, dim]
    and lse [n, heads] float32."""
    assert q.dim() == 3 and q.dtype in _TORCH_DT
    n, heads, dim = shape = q.shape
    device = torch.cuda.current_device()
    c = cache._with(table, n, device)
    assert dim == cache.dim, f"q: {cache.dim} dimensions expected"
    try:
        qp = _heads(q, shape, q.dtype, device, "q")
    except _Broadcast:
        return attention_step(cache, table, lengths, q.contiguous(), scale, longest, out)
    out, *op = _new_heads(q) if out is None else (out, *_heads(out, shape, q.dtype, device, "out"))
    lse = torch.empty((n, heads), dtype=torch.float32, device=q.device)
    _check(lib.fx_attention_step(c, n, _numbers(lengths, n, device, "lengths"), longest, _TORCH_DT[q.dtype], heads, dim ** -0.5 if scale is None else scale,
                                 *qp, *op, lse.data_ptr(), _stream()))
    return out, lse
