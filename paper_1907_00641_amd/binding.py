"""Thin Python binding of the C ABI in include/pam_lattice.h and
include/pam_attn.h (and the benchmark's row-copy probe in include/pam_probe.h).

Argument marshalling only: every step of the filter runs in the HIP
library ``libpam_lattice.so``.  PyTorch provides device memory and the
current stream; tensors are passed to the library as raw pointers.  There is
no fallback: if the library is not built, loading raises.
"""
from __future__ import annotations

import ctypes
import os

import torch

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libpam_lattice.so")

PAM_OK = 0
PAM_ERR_INVALID_ARGUMENT = 1
PAM_ERR_OUT_OF_MEMORY = 2
PAM_ERR_CAPACITY = 3
PAM_ERR_KEY_RANGE = 4
PAM_ERR_STATE = 5
PAM_ERR_DEVICE = 6
PAM_NORMALIZE = 1
PAM_EGRAD_AUGMENTED = 2
PAM_MAX_D = 16
PAM_MAX_C = 1024
PAM_MAX_GROUPS = 65536

# every symbol the header declares
EXPORTS = (
    "pam_lattice_build", "pam_filter_fwd", "pam_filter_bwd", "pam_lattice_stats",
    "pam_lattice_export", "pam_lattice_set_capacity", "pam_timing_enable", "pam_kernel_count",
    "pam_kernel_name", "pam_timing_read", "pam_lattice_destroy", "pam_status_string",
    "pam_last_error", "pam_lattice_build_groups", "pam_lattice_export_groups", "pam_filter_fwd_asym",
    "pam_filter_bwd_asym", "pam_block_fwd", "pam_block_bwd_workspace", "pam_block_bwd", "pam_block_bwd_noalloc",
    "pam_probe_copy_rows",
    "pam_diff_attn_fwd_workspace", "pam_diff_attn_bwd_workspace", "pam_diff_attn_fwd", "pam_diff_attn_bwd",
    "pam_rotary_frequencies", "pam_rotary_table", "pam_rotary", "pam_dropout", "pam_norm_gate_fwd",
    "pam_norm_gate_bwd_workspace", "pam_norm_gate_bwd",
)

# pam_dtype_t
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
PAM_ATTN_CAUSAL = 1
PAM_ROTARY_INTERLEAVED = 1
PAM_ROTARY_INVERSE = 2
ROPE_SCALINGS = {"plain": 0, "linear": 1, "ntk": 2, "yarn": 3}
NORMS = {"rms": 0, "layer": 1}


class BlockDesc(ctypes.Structure):
    """pam_block_desc_t of the C header."""
    _fields_ = [("c_in", ctypes.c_int32), ("d_tot", ctypes.c_int32), ("c_tot", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("dims", ctypes.c_int32 * 3), ("mesh_scale", ctypes.c_float),
                ("slope", ctypes.c_float)]


class DiffAttnDesc(ctypes.Structure):
    """pam_diff_attn_desc_t of the C header."""
    _fields_ = [("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("dim", ctypes.c_int32), ("dim_v", ctypes.c_int32),
                ("len_q", ctypes.c_int32), ("len_k", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("scale", ctypes.c_float), ("q_stride", ctypes.c_int64 * 4), ("k_stride", ctypes.c_int64 * 4),
                ("v_stride", ctypes.c_int64 * 3)]


class RotaryDesc(ctypes.Structure):
    """pam_rotary_desc_t of the C header."""
    _fields_ = [("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("length", ctypes.c_int32),
                ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("pairs", ctypes.c_int32), ("flags", ctypes.c_uint32), ("start", ctypes.c_int64),
                ("entries", ctypes.c_int64), ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3)]


class NormDesc(ctypes.Structure):
    """pam_norm_desc_t of the C header."""
    _fields_ = [("dtype", ctypes.c_int32), ("norm", ctypes.c_int32), ("rows", ctypes.c_int64),
                ("channels", ctypes.c_int32), ("eps", ctypes.c_float), ("gate_rows", ctypes.c_int64),
                ("x_stride", ctypes.c_int64), ("z_stride", ctypes.c_int64), ("p", ctypes.c_double),
                ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64)]

_lib = None
_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_i32 = ctypes.c_int32
_u32 = ctypes.c_uint32


class PamError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: {status_string(status)} ({detail})")
        self.status = status


def lib():
    """Load libpam_lattice.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built: run `python -m paper_1907_00641_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    L.pam_lattice_build.restype = ctypes.c_int
    L.pam_lattice_build.argtypes = [_vp, _i64, _i32, _vp, ctypes.POINTER(_vp)]
    L.pam_lattice_build_groups.restype = ctypes.c_int
    L.pam_lattice_build_groups.argtypes = [_vp, _i64, _i32, _vp, _i32, _vp, ctypes.POINTER(_vp)]
    L.pam_lattice_export_groups.restype = ctypes.c_int
    L.pam_lattice_export_groups.argtypes = [_vp, _vp]
    L.pam_filter_fwd.restype = ctypes.c_int
    L.pam_filter_fwd.argtypes = [_vp, _vp, _i32, _u32, _vp, _vp]
    L.pam_filter_fwd_asym.restype = ctypes.c_int
    L.pam_filter_fwd_asym.argtypes = [_vp, _i64, _vp, _i32, _u32, _vp, _vp]
    L.pam_filter_bwd_asym.restype = ctypes.c_int
    L.pam_filter_bwd_asym.argtypes = [_vp, _i64, _vp, _vp, _i32, _u32, _vp, _vp, _vp]
    L.pam_block_fwd.restype = ctypes.c_int
    L.pam_block_fwd.argtypes = [ctypes.POINTER(BlockDesc)] + [_vp] * 8
    L.pam_block_bwd_workspace.restype = ctypes.c_size_t
    L.pam_block_bwd_workspace.argtypes = [ctypes.POINTER(BlockDesc)]
    L.pam_block_bwd.restype = ctypes.c_int
    L.pam_block_bwd.argtypes = [ctypes.POINTER(BlockDesc)] + [_vp] * 13
    L.pam_block_bwd_noalloc.restype = ctypes.c_int
    L.pam_block_bwd_noalloc.argtypes = [ctypes.POINTER(BlockDesc)] + [_vp] * 12
    L.pam_filter_bwd.restype = ctypes.c_int
    L.pam_filter_bwd.argtypes = [_vp, _vp, _vp, _i32, _u32, _vp, _vp, _vp]
    L.pam_lattice_stats.restype = ctypes.c_int
    L.pam_lattice_stats.argtypes = [_vp, ctypes.POINTER(_i64), ctypes.POINTER(_i64)]
    L.pam_lattice_export.restype = ctypes.c_int
    L.pam_lattice_export.argtypes = [_vp, _vp, _vp, _vp, _vp]
    L.pam_lattice_set_capacity.restype = ctypes.c_int
    L.pam_lattice_set_capacity.argtypes = [_vp, _i64, _i32]
    L.pam_timing_enable.restype = ctypes.c_int
    L.pam_timing_enable.argtypes = [_vp, _i32]
    L.pam_kernel_count.restype = _i32
    L.pam_kernel_count.argtypes = []
    L.pam_kernel_name.restype = ctypes.c_char_p
    L.pam_kernel_name.argtypes = [_i32]
    L.pam_timing_read.restype = ctypes.c_int
    L.pam_timing_read.argtypes = [_vp, _i32, ctypes.POINTER(_i64), ctypes.POINTER(ctypes.c_double)]
    L.pam_probe_copy_rows.restype = ctypes.c_int
    L.pam_probe_copy_rows.argtypes = [_vp, _vp, _vp, _i64, _i32, _i32, _vp]
    L.pam_diff_attn_fwd_workspace.restype = ctypes.c_size_t
    L.pam_diff_attn_fwd_workspace.argtypes = [ctypes.POINTER(DiffAttnDesc)]
    L.pam_diff_attn_bwd_workspace.restype = ctypes.c_size_t
    L.pam_diff_attn_bwd_workspace.argtypes = [ctypes.POINTER(DiffAttnDesc)]
    L.pam_diff_attn_fwd.restype = ctypes.c_int
    L.pam_diff_attn_fwd.argtypes = [ctypes.POINTER(DiffAttnDesc)] + [_vp] * 12
    L.pam_diff_attn_bwd.restype = ctypes.c_int
    L.pam_diff_attn_bwd.argtypes = [ctypes.POINTER(DiffAttnDesc)] + [_vp] * 10 + [ctypes.POINTER(_i64)] + [_vp] * 6
    L.pam_rotary_frequencies.restype = ctypes.c_int
    L.pam_rotary_frequencies.argtypes = [_i32, ctypes.c_double, _i32] + [ctypes.c_double] * 4 + [_vp, _vp]
    L.pam_rotary_table.restype = ctypes.c_int
    L.pam_rotary_table.argtypes = [_vp, _vp, _vp, _i64, _i32, _i32, ctypes.c_double, _vp, _vp]
    L.pam_rotary.restype = ctypes.c_int
    L.pam_rotary.argtypes = [ctypes.POINTER(RotaryDesc)] + [_vp] * 7
    L.pam_dropout.restype = ctypes.c_int
    L.pam_dropout.argtypes = [_vp, _i64, _i32, ctypes.c_double, ctypes.c_uint64, ctypes.c_uint64, _vp, _vp]
    L.pam_norm_gate_fwd.restype = ctypes.c_int
    L.pam_norm_gate_fwd.argtypes = [ctypes.POINTER(NormDesc)] + [_vp] * 11
    L.pam_norm_gate_bwd_workspace.restype = ctypes.c_size_t
    L.pam_norm_gate_bwd_workspace.argtypes = [ctypes.POINTER(NormDesc)]
    L.pam_norm_gate_bwd.restype = ctypes.c_int
    L.pam_norm_gate_bwd.argtypes = [ctypes.POINTER(NormDesc)] + [_vp] * 19
    L.pam_lattice_destroy.restype = None
    L.pam_lattice_destroy.argtypes = [_vp]
    L.pam_status_string.restype = ctypes.c_char_p
    L.pam_status_string.argtypes = [ctypes.c_int]
    L.pam_last_error.restype = ctypes.c_char_p
    L.pam_last_error.argtypes = []
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().pam_status_string(status).decode()


def last_error() -> str:
    return lib().pam_last_error().decode()


def _check(status: int, where: str):
    if status != PAM_OK:
        raise PamError(status, where, last_error())


def _stream_ptr(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream)


def _dev_ptr(t: torch.Tensor | None, dtype, name: str) -> int | None:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


class Lattice:
    """A built lattice handle plus the borrowed feature tensor it reads."""

    def __init__(self, handle: int, feat: torch.Tensor, d: int):
        self.handle = ctypes.c_void_p(handle)
        self.feat = feat  # kept alive: the augmented-channel backward re-reads it
        self.n = feat.shape[0]
        self.d = d

    def __del__(self):
        if getattr(self, "handle", None) is not None and self.handle.value and _lib is not None:
            _lib.pam_lattice_destroy(self.handle)
            self.handle = None

    def destroy(self):
        if self.handle is not None and self.handle.value:
            lib().pam_lattice_destroy(self.handle)
        self.handle = None


def pam_lattice_build(feat: torch.Tensor, stream=None, lat: Lattice | None = None, group_start=None) -> Lattice:
    """Build (or rebuild in place) the lattice of ``feat`` (n x d fp32, device).
    ``group_start`` (G + 1 offsets, host) makes a batched build of G
    independent point groups (pam_lattice_build_groups)."""
    if feat.dim() != 2:
        raise ValueError("feat must be n x d")
    n, d = feat.shape
    ptr = _dev_ptr(feat, torch.float32, "feat")
    h = ctypes.c_void_p(lat.handle.value if lat is not None else None)
    if group_start is None:
        _check(lib().pam_lattice_build(ptr, n, d, _stream_ptr(stream), ctypes.byref(h)), "pam_lattice_build")
    else:
        import numpy as np

        gs = np.ascontiguousarray(np.asarray(group_start, dtype=np.int64))
        _check(lib().pam_lattice_build_groups(ptr, n, d, gs.ctypes.data, len(gs) - 1, _stream_ptr(stream),
                                              ctypes.byref(h)), "pam_lattice_build_groups")
    if lat is not None:
        lat.feat, lat.n, lat.d = feat, n, d
        return lat
    return Lattice(h.value, feat, d)


def pam_filter_fwd(lat: Lattice, val: torch.Tensor, flags: int = 0, out: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
    """Forward filter; returns ``out`` (n x C fp32, allocated if not given)."""
    if val.dim() != 2 or val.shape[0] != lat.n:
        raise ValueError("val must be n x C")
    if out is None:
        out = torch.empty_like(val)
    _check(lib().pam_filter_fwd(lat.handle, _dev_ptr(val, torch.float32, "val"), val.shape[1], flags,
                                _dev_ptr(out, torch.float32, "out"), _stream_ptr(stream)),
           "pam_filter_fwd")
    return out


def pam_filter_bwd(lat: Lattice, val: torch.Tensor, grad_out: torch.Tensor, flags: int = 0,
                   grad_val: torch.Tensor | bool | None = True, grad_feat: torch.Tensor | bool | None = True,
                   stream=None):
    """Backward filter; returns (grad_val, grad_feat), each None if skipped.
    Pass True to allocate an output, a tensor to fill it, None/False to skip."""
    if grad_val is True:
        grad_val = torch.empty_like(val)
    elif grad_val is False:
        grad_val = None
    if grad_feat is True:
        grad_feat = torch.empty_like(lat.feat)
    elif grad_feat is False:
        grad_feat = None
    _check(lib().pam_filter_bwd(lat.handle, _dev_ptr(val, torch.float32, "val"),
                                _dev_ptr(grad_out, torch.float32, "grad_out"), val.shape[1], flags,
                                _dev_ptr(grad_val, torch.float32, "grad_val"),
                                _dev_ptr(grad_feat, torch.float32, "grad_feat"), _stream_ptr(stream)),
           "pam_filter_bwd")
    return grad_val, grad_feat


def pam_filter_fwd_asym(lat: Lattice, n_keys: int, val: torch.Tensor, flags: int = 0,
                        out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Asymmetric forward filter over a lattice built on [keys; queries]:
    ``val`` holds the n_keys key values (n_keys x C); returns ``out`` for the
    n - n_keys queries."""
    if val.dim() != 2 or val.shape[0] != n_keys:
        raise ValueError("val must be n_keys x C")
    if out is None:
        out = torch.empty((lat.n - n_keys, val.shape[1]), dtype=val.dtype, device=val.device)
    _check(lib().pam_filter_fwd_asym(lat.handle, n_keys, _dev_ptr(val, torch.float32, "val"), val.shape[1], flags,
                                     _dev_ptr(out, torch.float32, "out"), _stream_ptr(stream)),
           "pam_filter_fwd_asym")
    return out


def pam_filter_bwd_asym(lat: Lattice, n_keys: int, val: torch.Tensor, grad_out: torch.Tensor, flags: int = 0,
                        grad_val: torch.Tensor | bool | None = True, grad_feat: torch.Tensor | bool | None = True,
                        stream=None):
    """Backward pass of the asymmetric filter; returns (grad_val (n_keys x C),
    grad_feat (n x d)), each None if skipped."""
    if grad_val is True:
        grad_val = torch.empty_like(val)
    elif grad_val is False:
        grad_val = None
    if grad_feat is True:
        grad_feat = torch.empty_like(lat.feat)
    elif grad_feat is False:
        grad_feat = None
    _check(lib().pam_filter_bwd_asym(lat.handle, n_keys, _dev_ptr(val, torch.float32, "val"),
                                     _dev_ptr(grad_out, torch.float32, "grad_out"), val.shape[1], flags,
                                     _dev_ptr(grad_val, torch.float32, "grad_val"),
                                     _dev_ptr(grad_feat, torch.float32, "grad_feat"), _stream_ptr(stream)),
           "pam_filter_bwd_asym")
    return grad_val, grad_feat


def block_desc(c_in: int, d_tot: int, c_tot: int, groups: int, dims, mesh_scale: float, slope: float) -> BlockDesc:
    return BlockDesc(c_in, d_tot, c_tot, groups, (ctypes.c_int32 * 3)(*dims), mesh_scale, slope)


def pam_block_fwd(desc: BlockDesc, x: torch.Tensor, wf: torch.Tensor, bf: torch.Tensor, wv: torch.Tensor,
                  bv: torch.Tensor, stream=None):
    """Permutohedral block prologue; returns (feat, val) in the grouped layout
    ((groups N) x d_tot/groups and (groups N) x c_tot/groups)."""
    n = desc.dims[0] * desc.dims[1] * desc.dims[2]
    G = desc.groups
    feat = torch.empty((G * n, desc.d_tot // G), dtype=torch.float32, device=x.device)
    val = torch.empty((G * n, desc.c_tot // G), dtype=torch.float32, device=x.device)
    f32 = torch.float32
    _check(lib().pam_block_fwd(ctypes.byref(desc), _dev_ptr(x, f32, "x"), _dev_ptr(wf, f32, "wf"),
                               _dev_ptr(bf, f32, "bf"), _dev_ptr(wv, f32, "wv"), _dev_ptr(bv, f32, "bv"),
                               feat.data_ptr(), val.data_ptr(), _stream_ptr(stream)), "pam_block_fwd")
    return feat, val


def pam_block_bwd(desc: BlockDesc, x: torch.Tensor, wf: torch.Tensor, bf: torch.Tensor, wv: torch.Tensor,
                  grad_feat: torch.Tensor, grad_val: torch.Tensor, stream=None):
    """Backward of the prologue; returns (grad_x, grad_wf, grad_bf, grad_wv, grad_bv)."""
    f32 = torch.float32
    outs = [torch.empty_like(x), torch.empty_like(wf), torch.empty_like(bf), torch.empty_like(wv),
            torch.empty((desc.c_tot,), dtype=f32, device=x.device)]
    ws_bytes = lib().pam_block_bwd_workspace(ctypes.byref(desc))
    ws = torch.empty((max(ws_bytes, 4) + 3) // 4, dtype=f32, device=x.device)
    _check(lib().pam_block_bwd(ctypes.byref(desc), _dev_ptr(x, f32, "x"), _dev_ptr(wf, f32, "wf"),
                               _dev_ptr(bf, f32, "bf"), _dev_ptr(wv, f32, "wv"),
                               _dev_ptr(grad_feat, f32, "grad_feat"), _dev_ptr(grad_val, f32, "grad_val"),
                               *[o.data_ptr() for o in outs], ws.data_ptr(), _stream_ptr(stream)), "pam_block_bwd")
    return tuple(outs)


def pam_block_bwd_noalloc(desc: BlockDesc, x: torch.Tensor, wf: torch.Tensor, bf: torch.Tensor, wv: torch.Tensor,
                          grad_feat: torch.Tensor, grad_val: torch.Tensor, out, stream=None):
    """pam_block_bwd through the allocation-free entry point: ``out`` is the
    caller's (grad_x, grad_wf, grad_bf, grad_wv, grad_bv), written in full."""
    f32 = torch.float32
    shapes = (tuple(x.shape), tuple(wf.shape), tuple(bf.shape), tuple(wv.shape), (desc.c_tot,))
    ptrs = [_dev_ptr(o, f32, name) for o, name in zip(out, ("grad_x", "grad_wf", "grad_bf", "grad_wv", "grad_bv"))]
    for o, shp in zip(out, shapes):
        if tuple(o.shape) != shp:
            raise ValueError(f"output of shape {tuple(o.shape)}, expected {shp}")
    _check(lib().pam_block_bwd_noalloc(ctypes.byref(desc), _dev_ptr(x, f32, "x"), _dev_ptr(wf, f32, "wf"),
                                       _dev_ptr(bf, f32, "bf"), _dev_ptr(wv, f32, "wv"),
                                       _dev_ptr(grad_feat, f32, "grad_feat"), _dev_ptr(grad_val, f32, "grad_val"),
                                       *ptrs, _stream_ptr(stream)), "pam_block_bwd_noalloc")
    return tuple(out)


def pam_lattice_stats(lat: Lattice):
    """Returns (num_vertices, table_capacity)."""
    m, cap = _i64(0), _i64(0)
    _check(lib().pam_lattice_stats(lat.handle, ctypes.byref(m), ctypes.byref(cap)), "pam_lattice_stats")
    return m.value, cap.value


def pam_lattice_export(lat: Lattice):
    """Host copies: keys (M x d), vert (n x (d+1)), bary (n x (d+1)), nbr (M x (d+1) x 2)."""
    import numpy as np

    M, _ = pam_lattice_stats(lat)
    d, n = lat.d, lat.n
    keys = np.zeros((M, d), dtype=np.int32)
    vert = np.zeros((n, d + 1), dtype=np.int32)
    bary = np.zeros((n, d + 1), dtype=np.float32)
    nbr = np.zeros((M, d + 1, 2), dtype=np.int32)
    _check(lib().pam_lattice_export(lat.handle, keys.ctypes.data, vert.ctypes.data, bary.ctypes.data,
                                    nbr.ctypes.data), "pam_lattice_export")
    return keys, vert, bary, nbr


def pam_lattice_export_groups(lat: Lattice):
    """Host copy of the group id of every vertex (M int32)."""
    import numpy as np

    M, _ = pam_lattice_stats(lat)
    vg = np.zeros(M, dtype=np.int32)
    if M:
        _check(lib().pam_lattice_export_groups(lat.handle, vg.ctypes.data), "pam_lattice_export_groups")
    return vg


def pam_lattice_set_capacity(lat: Lattice, table_capacity: int, allow_regrow: bool = True):
    _check(lib().pam_lattice_set_capacity(lat.handle, table_capacity, int(allow_regrow)),
           "pam_lattice_set_capacity")


def pam_timing_enable(lat: Lattice, enable: bool):
    _check(lib().pam_timing_enable(lat.handle, int(enable)), "pam_timing_enable")


def pam_kernel_names():
    L = lib()
    return [L.pam_kernel_name(k).decode() for k in range(L.pam_kernel_count())]


def pam_timing_read(lat: Lattice):
    """Synchronise; returns {kernel name: (launches, total_ms)}."""
    L = lib()
    res = {}
    for k, name in enumerate(pam_kernel_names()):
        cnt, ms = _i64(0), ctypes.c_double(0.0)
        _check(L.pam_timing_read(lat.handle, k, ctypes.byref(cnt), ctypes.byref(ms)), "pam_timing_read")
        if cnt.value:
            res[name] = (cnt.value, ms.value)
    return res


def pam_probe_copy_rows(src: torch.Tensor, dst: torch.Tensor, perm: torch.Tensor | None, mode: int,
                        stream=None):
    """Measurement utility: dst row (perm[i] if mode & 2 else i) = src row
    (perm[i] if mode & 1 else i) for the n rows of the n x c fp32 tensors."""
    if src.dim() != 2 or src.shape != dst.shape:
        raise ValueError("src and dst must be n x c tensors of one shape")
    n, c = src.shape
    ps = _dev_ptr(src, torch.float32, "src")
    pd = _dev_ptr(dst, torch.float32, "dst")
    pp = _dev_ptr(perm, torch.int32, "perm") if mode else None
    if mode and perm.numel() != n:
        raise ValueError("perm must hold n entries")
    _check(lib().pam_probe_copy_rows(ps, pd, pp, n, c, mode, _stream_ptr(stream)), "pam_probe_copy_rows")


def pam_lattice_destroy(lat: Lattice):
    lat.destroy()


# ---------------------------------------------------------------------------
# the operators around an attention layer (include/pam_attn.h)
# ---------------------------------------------------------------------------

def _dtype_of(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32, float16 or bfloat16")
    return _DTYPES[t.dtype]


def _device_of(t: torch.Tensor, name: str) -> int:
    """Number of the current device, which ``t`` must be on."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a device tensor")
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"{name} must be on the current device")
    return dev


def _rows_ptr(t: torch.Tensor, dtype, dev: int, name: str) -> int:
    """Pointer of a strided tensor whose last axis is contiguous."""
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name} must be a device tensor of {dtype} on device {dev}")
    if t.stride(-1) != 1 and t.numel() and t.shape[-1] > 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return t.data_ptr()


def _shaped_ptr(t: torch.Tensor | None, shape, dtype, dev: int, name: str) -> int | None:
    """Pointer of a contiguous tensor of the given shape and type (None: NULL)."""
    if t is None:
        return None
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name} must be a device tensor of {dtype} on device {dev}")
    raise ValueError(f"{name} must be contiguous")


def _counts(*n: int):
    """Refuses sizes that the C ABI's 32-bit fields would take modulo 2^32."""
    if max(n) > 0x7FFFFFFF:
        raise ValueError("a size is 2^31 or more")


def _new(stream, make):
    """What ``make`` allocates, on the stream that writes it: memory freed after the
    call is not handed out again while that stream uses it."""
    if stream is None:
        return make()
    with torch.cuda.stream(stream):
        return make()


_SIZE_MAX = ctypes.c_size_t(-1).value


def _workspace_bytes(n: int, where: str) -> int:
    if n == _SIZE_MAX:
        raise PamError(PAM_ERR_INVALID_ARGUMENT, where, last_error())
    return n


def _diff_attn_desc(q, k, v, lam, scale, causal, q_len, k_len, key_mask):
    """Descriptor of a call and the pointers that both directions take."""
    if q.dim() != 5 or q.shape[3] != 2 or k.dim() != 5 or k.shape[3] != 2 or v.dim() != 4:
        raise ValueError("q must be B x Lq x H x 2 x d, k B x Lk x Hk x 2 x d, v B x Lk x Hk x dv")
    B, lq, H, _, d = q.shape
    _, lk, hk, dv = v.shape
    if k.shape != (B, lk, hk, 2, d) or v.shape[0] != B:
        raise ValueError("q, k and v do not agree in sequences, lengths, key heads or head size")
    _counts(B, lq, lk, H, hk, d, dv)
    dt = q.dtype
    code, dev = _dtype_of(q, "q"), _device_of(q, "q")
    ptrs = [_rows_ptr(q, dt, dev, "q"), _rows_ptr(k, dt, dev, "k"), _rows_ptr(v, dt, dev, "v"),
            _shaped_ptr(lam, (H,), dt, dev, "lam"), _shaped_ptr(q_len, (B,), torch.int32, dev, "q_len"),
            _shaped_ptr(k_len, (B,), torch.int32, dev, "k_len"), None]
    if key_mask is not None:
        if key_mask.dtype not in (torch.bool, torch.uint8):
            raise ValueError("key_mask must be bool or uint8")
        ptrs[6] = _shaped_ptr(key_mask, (B, lk), key_mask.dtype, dev, "key_mask")
    desc = DiffAttnDesc(code, B, H, hk, d, dv, lq, lk, PAM_ATTN_CAUSAL if causal else 0,
                        d ** -0.5 if scale is None else scale, q.stride()[:4], k.stride()[:4], v.stride()[:3])
    return desc, ptrs, dev


def pam_diff_attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lam: torch.Tensor, *,
                      scale: float | None = None, causal: bool = False, q_len: torch.Tensor | None = None,
                      k_len: torch.Tensor | None = None, key_mask: torch.Tensor | None = None, save: bool = False,
                      stream=None):
    """Differential attention, out = (P1 - lam P2) v per head.

    ``q`` is B x Lq x H x 2 x d, ``k`` B x Lk x Hk x 2 x d, ``v`` B x Lk x Hk x dv (any strides, last axis
    contiguous), ``lam`` H values of q's type; ``scale`` 1 / sqrt(d) if not given; ``q_len``, ``k_len`` B int32
    and ``key_mask`` B x Lk (bool or uint8) on the device.  Returns ``out`` (B x Lq x H x dv); with ``save``
    (out, saved), saved being what pam_diff_attn_bwd takes."""
    desc, ptrs, _ = _diff_attn_desc(q, k, v, lam, scale, causal, q_len, k_len, key_mask)
    L, d = lib(), ctypes.byref(desc)
    shape = (*q.shape[:3], v.shape[3])
    ws_bytes = _workspace_bytes(L.pam_diff_attn_fwd_workspace(d), "pam_diff_attn_fwd")

    def make():
        out = q.new_empty(shape)
        so = q.new_empty((2, *shape), dtype=torch.float32) if save else None
        lse = q.new_empty((2, shape[0], shape[2], shape[1]), dtype=torch.float32) if save else None
        return out, so, lse, q.new_empty(ws_bytes, dtype=torch.uint8) if ws_bytes else None

    out, so, lse, ws = _new(stream, make)
    _check(L.pam_diff_attn_fwd(d, *ptrs, out.data_ptr(), so.data_ptr() if save else None,
                               lse.data_ptr() if save else None, ws.data_ptr() if ws_bytes else None,
                               _stream_ptr(stream)), "pam_diff_attn_fwd")
    return (out, (so, lse)) if save else out


def pam_diff_attn_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lam: torch.Tensor, saved,
                      grad_out: torch.Tensor, *, scale: float | None = None, causal: bool = False,
                      q_len: torch.Tensor | None = None, k_len: torch.Tensor | None = None,
                      key_mask: torch.Tensor | None = None, stream=None):
    """Gradients (q, k, v, lam) of pam_diff_attn_fwd with the same arguments,
    from its ``saved`` and ``grad_out`` (B x Lq x H x dv, any strides)."""
    desc, ptrs, dev = _diff_attn_desc(q, k, v, lam, scale, causal, q_len, k_len, key_mask)
    L, d = lib(), ctypes.byref(desc)
    shape = (*q.shape[:3], v.shape[3])
    so, lse = saved
    pso = _shaped_ptr(so, (2, *shape), torch.float32, dev, "saved o")
    plse = _shaped_ptr(lse, (2, shape[0], shape[2], shape[1]), torch.float32, dev, "saved lse")
    if grad_out.shape != shape:
        raise ValueError(f"grad_out has shape {tuple(grad_out.shape)}, expected {shape}")
    pdo = _rows_ptr(grad_out, q.dtype, dev, "grad_out")
    ws_bytes = _workspace_bytes(L.pam_diff_attn_bwd_workspace(d), "pam_diff_attn_bwd")
    gq, gk, gv, gl, ws = _new(stream, lambda: (
        q.new_empty(q.shape), q.new_empty(k.shape), q.new_empty(v.shape), q.new_empty(lam.shape),
        q.new_empty(max(ws_bytes, 16), dtype=torch.uint8)))
    _check(L.pam_diff_attn_bwd(d, *ptrs, pso, plse, pdo, (_i64 * 3)(*grad_out.stride()[:3]), gq.data_ptr(),
                               gk.data_ptr(), gv.data_ptr(), gl.data_ptr(), ws.data_ptr(), _stream_ptr(stream)),
           "pam_diff_attn_bwd")
    return gq, gk, gv, gl


def pam_rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                           original_len: float = 0.0, beta_slow: float = 1.0, beta_fast: float = 32.0):
    """Angles per unit of position of the rot / 2 pairs (CPU float64) and the factor of cosines and sines;
    ``scaling`` "plain", "linear", "ntk" or "yarn" for contexts longer than the trained one."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(ROPE_SCALINGS)}")
    _counts(rot)
    freq = torch.empty(max(rot // 2, 1), dtype=torch.float64)
    mag = ctypes.c_double(0.0)
    _check(lib().pam_rotary_frequencies(rot, base, ROPE_SCALINGS[scaling], factor, original_len, beta_slow, beta_fast,
                                        freq.data_ptr(), ctypes.byref(mag)), "pam_rotary_frequencies")
    return freq, mag.value


def pam_rotary_table(freq: torch.Tensor, entries: int | None = None, coord: torch.Tensor | None = None,
                     axis: torch.Tensor | None = None, magnitude: float = 1.0, stream=None) -> torch.Tensor:
    """Table (entries x pairs x 2 fp32) of the cosines and sines of freq[i] times the entry's number, or times
    coord[t, axis[i]] (``coord`` entries x axes fp32, ``axis`` pairs int32)."""
    if freq.dim() != 1:
        raise ValueError("freq must have one axis")
    pairs, axes = freq.shape[0], 1
    if coord is not None:
        if coord.dim() != 2:
            raise ValueError("coord must be entries x axes")
        if entries is not None and entries != coord.shape[0]:
            raise ValueError("entries is not the number of coordinates")
        entries, axes = coord.shape
    elif entries is None:
        raise ValueError("give entries or coord")
    _counts(pairs, axes)
    dev = _device_of(freq, "freq")
    pf = _shaped_ptr(freq, (pairs,), torch.float64, dev, "freq")
    pc = _shaped_ptr(coord, (entries, axes), torch.float32, dev, "coord")
    pa = _shaped_ptr(axis, (pairs,), torch.int32, dev, "axis")
    table = _new(stream, lambda: freq.new_empty((max(entries, 0), pairs, 2), dtype=torch.float32))
    _check(lib().pam_rotary_table(pf, pc, pa, entries, pairs, axes, magnitude, table.data_ptr(),
                                  _stream_ptr(stream)), "pam_rotary_table")
    return table


def pam_rotary(q: torch.Tensor, k: torch.Tensor | None, table: torch.Tensor, *, pos: torch.Tensor | None = None,
               start: int = 0, interleaved: bool = False, inverse: bool = False, out=None, stream=None):
    """Rotates the first 2 pairs channels of the heads of ``q`` (B x L x H x d) and ``k`` (B x L x Hk x d, or
    None) by ``table`` (entries x pairs x 2); token l takes entry pos[b, l] (B x L int32) or start + l.
    ``inverse`` rotates back (gradients).  ``out`` = (q_out, k_out), contiguous; contiguous inputs may be their
    own outputs.  Returns (q', k')."""
    if q.dim() != 4 or (k is not None and (k.dim() != 4 or k.shape[:2] != q.shape[:2] or k.shape[3] != q.shape[3])):
        raise ValueError("q must be B x L x H x d and k B x L x Hk x d")
    if table.dim() != 3 or table.shape[2] != 2:
        raise ValueError("table must be entries x pairs x 2")
    B, n, H, d = q.shape
    hk = 0 if k is None else k.shape[2]
    _counts(B, n, H, hk, d, table.shape[1])
    if not -(1 << 62) < start < 1 << 62:
        raise ValueError("start must be less than 2^62 in size")
    flags = (PAM_ROTARY_INTERLEAVED if interleaved else 0) | (PAM_ROTARY_INVERSE if inverse else 0)
    desc = RotaryDesc(_dtype_of(q, "q"), B, n, H, hk, d, table.shape[1], flags, start, table.shape[0],
                      q.stride()[:3], (0, 0, 0) if k is None else k.stride()[:3])
    dt, dev = q.dtype, _device_of(q, "q")
    pq, pk = _rows_ptr(q, dt, dev, "q"), None if k is None else _rows_ptr(k, dt, dev, "k")
    pt = _shaped_ptr(table, table.shape, torch.float32, dev, "table")
    pp = _shaped_ptr(pos, (B, n), torch.int32, dev, "pos")
    if out is None:
        qo, ko = _new(stream, lambda: (q.new_empty(q.shape), None if k is None else q.new_empty(k.shape)))
        pqo, pko = qo.data_ptr(), None if k is None else ko.data_ptr()
    else:
        qo, ko = out
        pqo = _shaped_ptr(qo, q.shape, dt, dev, "q_out")
        pko = None if k is None else _shaped_ptr(ko, k.shape, dt, dev, "k_out")
    _check(lib().pam_rotary(ctypes.byref(desc), pq, pk, pt, pp, pqo, pko, _stream_ptr(stream)), "pam_rotary")
    return qo, ko


def pam_dropout(x: torch.Tensor, p: float, seed: int, offset: int = 0, out: torch.Tensor | None = None,
                stream=None) -> torch.Tensor:
    """x times 1 / (1 - p) where the numbers that Philox4x32-10 makes of (seed, offset, element) keep it, else 0.
    The gradient is the same call on the upstream gradient.  ``out`` may be ``x``."""
    code, dev = _dtype_of(x, "x"), _device_of(x, "x")
    px = _shaped_ptr(x, x.shape, x.dtype, dev, "x")
    if out is None:
        out = _new(stream, lambda: x.new_empty(x.shape))
        po = out.data_ptr()
    else:
        po = _shaped_ptr(out, x.shape, x.dtype, dev, "out")
    _check(lib().pam_dropout(px, x.numel(), code, p, seed, offset, po, _stream_ptr(stream)), "pam_dropout")
    return out


def _norm_desc(x, z, w_post, b_post, gate, scale, w_pre, b_pre, norm, eps, p, seed, offset):
    if x.dim() != 2 or (z is not None and z.shape != x.shape):
        raise ValueError("x and z must be rows x channels")
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {sorted(NORMS)}")
    n, c = x.shape
    _counts(c)
    gate_rows = 0
    if gate is not None:
        if gate.dim() != 2 or gate.shape[1] != c or (gate.shape[0] == 0) != (n == 0) or \
                (gate.shape[0] and n % gate.shape[0]):
            raise ValueError("gate must be rows x channels, its rows dividing x's")
        gate_rows = n // gate.shape[0] if gate.shape[0] else 1
    dt, f32 = x.dtype, torch.float32
    desc = NormDesc(_dtype_of(x, "x"), NORMS[norm], n, c, eps, gate_rows, x.stride(0),
                    x.stride(0) if z is None else z.stride(0), p, seed, offset)
    dev = _device_of(x, "x")
    ptrs = [_rows_ptr(x, dt, dev, "x"), None if z is None else _rows_ptr(z, dt, dev, "z"),
            _shaped_ptr(w_post, (c,), f32, dev, "w_post"), _shaped_ptr(b_post, (c,), f32, dev, "b_post"),
            None if gate is None else _shaped_ptr(gate, gate.shape, dt, dev, "gate"),
            _shaped_ptr(scale, (c,), f32, dev, "scale"), _shaped_ptr(w_pre, (c,), f32, dev, "w_pre"),
            _shaped_ptr(b_pre, (c,), f32, dev, "b_pre")]
    return desc, ptrs, dev


def pam_norm_gate_fwd(x: torch.Tensor, *, z: torch.Tensor | None = None, w_post: torch.Tensor | None = None,
                      b_post: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                      scale: torch.Tensor | None = None, w_pre: torch.Tensor | None = None,
                      b_pre: torch.Tensor | None = None, norm: str = "rms", eps: float = 1e-6, p: float = 0.0,
                      seed: int = 0, offset: int = 0, next_norm: bool = True, stream=None):
    """r = x + drop(scale gate (N(z) w_post + b_post)) and h = N(r) w_pre + b_pre, in one pass over the rows.

    ``x``, ``z`` rows x channels (``z`` None: r is x), ``gate`` G x channels (each row for rows / G consecutive
    rows), vectors fp32.  Returns (r, h); r is None without z, h without ``next_norm``."""
    desc, ptrs, _ = _norm_desc(x, z, w_post, b_post, gate, scale, w_pre, b_pre, norm, eps, p, seed, offset)
    r, h = _new(stream, lambda: (None if z is None else x.new_empty(x.shape),
                                 x.new_empty(x.shape) if next_norm else None))
    _check(lib().pam_norm_gate_fwd(ctypes.byref(desc), *ptrs, None if r is None else r.data_ptr(),
                                   None if h is None else h.data_ptr(), _stream_ptr(stream)), "pam_norm_gate_fwd")
    return r, h


def pam_norm_gate_bwd(x: torch.Tensor, *, grad_r: torch.Tensor | None, grad_h: torch.Tensor | None,
                      z: torch.Tensor | None = None, w_post: torch.Tensor | None = None,
                      b_post: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                      scale: torch.Tensor | None = None, w_pre: torch.Tensor | None = None,
                      b_pre: torch.Tensor | None = None, norm: str = "rms", eps: float = 1e-6, p: float = 0.0,
                      seed: int = 0, offset: int = 0, stream=None) -> dict:
    """Gradients of pam_norm_gate_fwd with the same arguments, by the arguments' names (None for those not
    given), from ``grad_r`` (None: 0) and ``grad_h`` (None: the forward call had no next norm)."""
    desc, ptrs, dev = _norm_desc(x, z, w_post, b_post, gate, scale, w_pre, b_pre, norm, eps, p, seed, offset)
    L, d = lib(), ctypes.byref(desc)
    pr = _shaped_ptr(grad_r, x.shape, x.dtype, dev, "grad_r")
    ph = _shaped_ptr(grad_h, x.shape, x.dtype, dev, "grad_h")
    ws_bytes = _workspace_bytes(L.pam_norm_gate_bwd_workspace(d), "pam_norm_gate_bwd")
    given = (x, z, w_post, b_post, gate, scale, w_pre, b_pre)
    *grads, ws = _new(stream, lambda: [None if t is None else t.new_empty(t.shape) for t in given] + [
        x.new_empty(max(ws_bytes, 16), dtype=torch.uint8)])
    _check(L.pam_norm_gate_bwd(d, *ptrs[:7], pr, ph, *(None if t is None else t.data_ptr() for t in grads),
                               ws.data_ptr(), _stream_ptr(stream)), "pam_norm_gate_bwd")
    return dict(zip(("x", "z", "w_post", "b_post", "gate", "scale", "w_pre", "b_pre"), grads))
