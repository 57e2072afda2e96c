"""ctypes binding of libbsa.so: argument marshalling only.

Every step of the path runs in the library's HIP kernels; PyTorch supplies device
memory (tensors) and the stream.  The functions mirror the C ABI of include/bsa.h
name for name (without the `bsa_` prefix) and raise BsaError on a negative status.
Importing this module fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from math import sqrt
from typing import Optional

import torch

# BSA_LIB selects another build of the same library (e.g. one compiled with different tuning flags)
_LIB_PATH = os.environ.get("BSA_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbsa.so")

F32, BF16 = 0, 1
RASTER, BLOCK_MAJOR = 0, 1
EXPORTS = (
    "bsa_strerror", "bsa_n_keep", "bsa_pool_blocks", "bsa_select_workspace_bytes", "bsa_select_kv",
    "bsa_select_kv_stat", "bsa_select_kv_static", "bsa_prune_q", "bsa_fwd_workspace_bytes", "bsa_attn_fwd", "bsa_bwd_workspace_bytes", "bsa_attn_bwd", "bsa_attn_bwd_stages",
    "bsa_dense_bwd_workspace_bytes", "bsa_dense_attn_fwd", "bsa_dense_attn_bwd", "bsa_mfma_probe",
    "bsa_rope_table_bytes", "bsa_rope_table", "bsa_qk_norm_rope_fwd", "bsa_qk_norm_rope_bwd_workspace_bytes", "bsa_qk_norm_rope_bwd",
    "bsa_cross_attn_fwd_workspace_bytes", "bsa_cross_attn_fwd", "bsa_cross_attn_bwd_workspace_bytes", "bsa_cross_attn_bwd",
)


class BsaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {lib().bsa_strerror(status).decode()} (status {status})")


class ShapeStruct(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "H", "T", "Hs", "Ws", "Ct", "Ch", "Cw", "d", "dtype", "Wt", "Wh", "Ww", "layout")]


class StridesStruct(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("b", "l", "h")]


class RopeStruct(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dt", "dh", "dw", "style")]


class CrossStruct(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "H", "Hkv", "Lq", "S", "d", "dtype")] + [(n, StridesStruct) for n in "qkvo"]


# the same from one pack: field by field they take longer to fill than a small call to launch
_CROSS, _FOUR, _FOUR_STRIDES = struct.Struct("7i4x12q"), struct.Struct("12q"), StridesStruct * 4

_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2509_01085_amd.build` "
                "(there is no fallback path)")
        L = C.CDLL(_LIB_PATH)
        P, vp, i32, i64, f32, f64, sz = C.POINTER(ShapeStruct), C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_double, C.c_size_t
        L.bsa_strerror.restype, L.bsa_strerror.argtypes = C.c_char_p, [C.c_int]
        L.bsa_n_keep.restype, L.bsa_n_keep.argtypes = C.c_int, [P, f64]
        L.bsa_pool_blocks.restype, L.bsa_pool_blocks.argtypes = C.c_int, [P, vp, vp, vp]
        L.bsa_select_workspace_bytes.restype, L.bsa_select_workspace_bytes.argtypes = sz, [P]
        L.bsa_select_kv.restype = C.c_int
        L.bsa_select_kv.argtypes = [P, vp, vp, f64, f64, vp, vp, i64, vp, vp, vp, vp, sz, vp]
        L.bsa_select_kv_stat.restype = C.c_int
        L.bsa_select_kv_stat.argtypes = [P, vp, vp, f64, f64, f64, vp, vp, i64, vp, vp, vp, vp, sz, vp]
        L.bsa_select_kv_static.restype = C.c_int
        L.bsa_select_kv_static.argtypes = [P, vp, vp, f64, f64, vp, vp, i64, vp, vp, vp, vp]
        L.bsa_prune_q.restype, L.bsa_prune_q.argtypes = C.c_int, [P, vp, f64, vp, vp]
        L.bsa_attn_fwd.restype = C.c_int
        L.bsa_attn_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, i32, f32, vp, vp, vp, sz, vp]
        L.bsa_fwd_workspace_bytes.restype, L.bsa_fwd_workspace_bytes.argtypes = sz, [P, i32]
        L.bsa_bwd_workspace_bytes.restype, L.bsa_bwd_workspace_bytes.argtypes = sz, [P, i32]
        L.bsa_attn_bwd.restype = C.c_int
        L.bsa_attn_bwd.argtypes = [P] + [vp] * 11 + [i32, f32, vp, vp, vp, vp, sz, vp]
        L.bsa_attn_bwd_stages.restype = C.c_int
        L.bsa_attn_bwd_stages.argtypes = [P] + [vp] * 11 + [i32, f32, vp, vp, vp, vp, sz, C.c_uint, vp]
        L.bsa_dense_bwd_workspace_bytes.restype, L.bsa_dense_bwd_workspace_bytes.argtypes = sz, [P]
        L.bsa_dense_attn_fwd.restype = C.c_int
        L.bsa_dense_attn_fwd.argtypes = [P, vp, vp, vp, f32, vp, vp, vp]
        L.bsa_dense_attn_bwd.restype = C.c_int
        L.bsa_dense_attn_bwd.argtypes = [P] + [vp] * 6 + [f32, vp, vp, vp, vp, sz, vp]
        R, T, X = C.POINTER(RopeStruct), C.POINTER(StridesStruct), C.POINTER(CrossStruct)
        L.bsa_rope_table_bytes.restype, L.bsa_rope_table_bytes.argtypes = sz, [P, R]
        L.bsa_rope_table.restype, L.bsa_rope_table.argtypes = C.c_int, [P, R, f64, i64, i64, i64, vp, vp]
        L.bsa_qk_norm_rope_fwd.restype = C.c_int
        L.bsa_qk_norm_rope_fwd.argtypes = [P, R] + [vp] * 4 + [T, vp, vp, f32] + [vp] * 4
        L.bsa_qk_norm_rope_bwd_workspace_bytes.restype, L.bsa_qk_norm_rope_bwd_workspace_bytes.argtypes = sz, [P]
        L.bsa_qk_norm_rope_bwd.restype = C.c_int
        L.bsa_qk_norm_rope_bwd.argtypes = [P, R] + [vp] * 3 + [T, vp, vp, f32] + [vp] * 6 + [T, vp, vp, vp, sz, vp]
        L.bsa_cross_attn_fwd_workspace_bytes.restype, L.bsa_cross_attn_fwd_workspace_bytes.argtypes = sz, [X]
        L.bsa_cross_attn_fwd.restype, L.bsa_cross_attn_fwd.argtypes = C.c_int, [X] + [vp] * 5 + [f32, vp, vp, vp, sz, vp]
        L.bsa_cross_attn_bwd_workspace_bytes.restype, L.bsa_cross_attn_bwd_workspace_bytes.argtypes = sz, [X]
        L.bsa_cross_attn_bwd.restype = C.c_int
        L.bsa_cross_attn_bwd.argtypes = [X] + [vp] * 8 + [f32] + [vp] * 3 + [T, vp, sz, vp]
        L.bsa_mfma_probe.restype, L.bsa_mfma_probe.argtypes = i64, [i32, i32, vp, vp]
        _lib = L
    return _lib


@dataclass(frozen=True)
class Shape:
    B: int
    H: int
    T: int
    Hs: int
    Ws: int
    Ct: int
    Ch: int
    Cw: int
    d: int
    dtype: int  # F32 or BF16
    Wt: int = 0  # window of the critical-token mechanism; 0, 0, 0 = the whole block
    Wh: int = 0
    Ww: int = 0
    layout: int = 0  # RASTER or BLOCK_MAJOR

    @property
    def L(self) -> int:
        return self.T * self.Hs * self.Ws

    @property
    def Bk(self) -> int:
        return self.Ct * self.Ch * self.Cw

    @property
    def N(self) -> int:
        return self.L // self.Bk

    @property
    def rows(self) -> int:
        return self.B * self.H * self.N

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == F32 else torch.bfloat16

    def c(self) -> ShapeStruct:
        return ShapeStruct(self.B, self.H, self.T, self.Hs, self.Ws, self.Ct, self.Ch, self.Cw, self.d, self.dtype,
                           self.Wt, self.Wh, self.Ww, self.layout)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "libbsa takes contiguous tensors"
    return t.data_ptr()


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _check(status: int, where: str) -> None:
    if status < 0:
        raise BsaError(status, where)


def n_keep(shape: Shape, keep_ratio: float) -> int:
    n = lib().bsa_n_keep(C.byref(shape.c()), keep_ratio)
    _check(n, "bsa_n_keep")
    return n


def pool_blocks(shape: Shape, X: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    if out is None:
        out = torch.empty((shape.B, shape.H, shape.N, shape.d), dtype=torch.float64, device=X.device)
    _check(lib().bsa_pool_blocks(C.byref(shape.c()), _ptr(X), _ptr(out), _stream()), "bsa_pool_blocks")
    return out


@dataclass
class KvLists:
    q2k_ptr: torch.Tensor  # [rows+1] int32
    q2k_idx: torch.Tensor  # [rows*N] int32 (first nnz valid)
    k2q_ptr: Optional[torch.Tensor]
    k2q_idx: Optional[torch.Tensor]
    nnz: torch.Tensor  # int64 device scalar
    workspace: torch.Tensor


def select_workspace_bytes(shape: Shape) -> int:
    return lib().bsa_select_workspace_bytes(C.byref(shape.c()))


STATIC_SELECT_BYTES = 32 << 20  # BSA_STATIC_SELECT_BYTES of the header


def alloc_kv_lists(shape: Shape, device, transpose: bool = True, workspace: bool = True) -> KvLists:
    cap = shape.rows * shape.N
    i32 = dict(dtype=torch.int32, device=device)
    return KvLists(
        torch.empty(shape.rows + 1, **i32), torch.empty(cap, **i32),
        torch.empty(shape.rows + 1, **i32) if transpose else None,
        torch.empty(cap, **i32) if transpose else None,
        torch.zeros(1, dtype=torch.int64, device=device),
        torch.empty(select_workspace_bytes(shape) if workspace else 0, dtype=torch.uint8, device=device))


def select_kv_static(shape: Shape, Qbar: torch.Tensor, Kbar: torch.Tensor, threshold: float, out: KvLists,
                     score_scale: Optional[float] = None) -> KvLists:
    """bsa_select_kv_static: the selection with the library's built-in scratch; `out` (lists and
    the nnz scalar, no workspace needed) comes from the caller, the call allocates nothing."""
    if score_scale is None:
        score_scale = 1.0 / sqrt(shape.d)
    st = lib().bsa_select_kv_static(C.byref(shape.c()), _ptr(Qbar), _ptr(Kbar), threshold, score_scale,
                                    _ptr(out.q2k_ptr), _ptr(out.q2k_idx), out.q2k_idx.numel(), _ptr(out.k2q_ptr),
                                    _ptr(out.k2q_idx), _ptr(out.nnz), _stream())
    _check(st, "bsa_select_kv_static")
    return out


def select_kv(shape: Shape, Qbar: torch.Tensor, Kbar: torch.Tensor, threshold: float,
              score_scale: Optional[float] = None, out: Optional[KvLists] = None,
              transpose: bool = True, stat_z: Optional[float] = None) -> KvLists:
    """stat_z: the quantile U(1 - k/n) of Eq. 3, supplied by the caller; None = plain Eq. 4."""
    if out is None:
        out = alloc_kv_lists(shape, Qbar.device, transpose)
    if score_scale is None:
        score_scale = 1.0 / sqrt(shape.d)
    tail = (_ptr(out.q2k_ptr), _ptr(out.q2k_idx), out.q2k_idx.numel(), _ptr(out.k2q_ptr), _ptr(out.k2q_idx),
            _ptr(out.nnz), _ptr(out.workspace), out.workspace.numel(), _stream())
    if stat_z is None:
        st = lib().bsa_select_kv(C.byref(shape.c()), _ptr(Qbar), _ptr(Kbar), threshold, score_scale, *tail)
    else:
        st = lib().bsa_select_kv_stat(C.byref(shape.c()), _ptr(Qbar), _ptr(Kbar), threshold, stat_z, score_scale, *tail)
    _check(st, "bsa_select_kv")
    return out


def prune_q(shape: Shape, Q: torch.Tensor, keep_ratio: float, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    nk = n_keep(shape, keep_ratio)
    if out is None:
        out = torch.empty((shape.B, shape.H, shape.N, nk), dtype=torch.int32, device=Q.device)
    _check(lib().bsa_prune_q(C.byref(shape.c()), _ptr(Q), keep_ratio, _ptr(out), _stream()), "bsa_prune_q")
    return out


def fwd_workspace_bytes(shape: Shape, n_keep_: int) -> int:
    return lib().bsa_fwd_workspace_bytes(C.byref(shape.c()), n_keep_)


def attn_fwd(shape: Shape, Q, K, V, lists: KvLists, keep_idx: torch.Tensor, sm_scale: Optional[float] = None,
             O: Optional[torch.Tensor] = None, LSE: Optional[torch.Tensor] = None,
             workspace: Optional[torch.Tensor] = None):
    nk = keep_idx.shape[-1]
    if workspace is None:
        workspace = torch.empty(max(1, fwd_workspace_bytes(shape, nk)), dtype=torch.uint8, device=Q.device)
    if sm_scale is None:
        sm_scale = 1.0 / sqrt(shape.d)
    if O is None:
        O = torch.empty_like(Q)
    if LSE is None:
        LSE = torch.empty((shape.B, shape.H, shape.L), dtype=torch.float32, device=Q.device)
    st = lib().bsa_attn_fwd(C.byref(shape.c()), _ptr(Q), _ptr(K), _ptr(V), _ptr(lists.q2k_ptr), _ptr(lists.q2k_idx),
                            _ptr(keep_idx), nk, sm_scale, _ptr(O), _ptr(LSE), _ptr(workspace), workspace.numel(),
                            _stream())
    _check(st, "bsa_attn_fwd")
    return O, LSE


def bwd_workspace_bytes(shape: Shape, n_keep_: int) -> int:
    return lib().bsa_bwd_workspace_bytes(C.byref(shape.c()), n_keep_)


BWD_PRE, BWD_DQ, BWD_DKV = 1, 2, 4


def attn_bwd(shape: Shape, Q, K, V, O, LSE, dO, lists: KvLists, keep_idx: torch.Tensor,
             sm_scale: Optional[float] = None, dQ=None, dK=None, dV=None, workspace: Optional[torch.Tensor] = None,
             stages: Optional[int] = None):
    if sm_scale is None:
        sm_scale = 1.0 / sqrt(shape.d)
    nk = keep_idx.shape[-1]
    dQ = torch.empty_like(Q) if dQ is None else dQ
    dK = torch.empty_like(K) if dK is None else dK
    dV = torch.empty_like(V) if dV is None else dV
    if workspace is None:
        workspace = torch.empty(max(1, bwd_workspace_bytes(shape, nk)), dtype=torch.uint8, device=Q.device)
    args = (C.byref(shape.c()), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(dO),
            _ptr(lists.q2k_ptr), _ptr(lists.q2k_idx), _ptr(lists.k2q_ptr), _ptr(lists.k2q_idx),
            _ptr(keep_idx), nk, sm_scale, _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(workspace), workspace.numel())
    if stages is None:
        st = lib().bsa_attn_bwd(*args, _stream())
    else:
        st = lib().bsa_attn_bwd_stages(*args, stages, _stream())
    _check(st, "bsa_attn_bwd")
    return dQ, dK, dV


def dense_bwd_workspace_bytes(shape: Shape) -> int:
    return lib().bsa_dense_bwd_workspace_bytes(C.byref(shape.c()))


def dense_attn_fwd(shape: Shape, Q, K, V, sm_scale: Optional[float] = None, O=None, LSE=None):
    if sm_scale is None:
        sm_scale = 1.0 / sqrt(shape.d)
    O = torch.empty_like(Q) if O is None else O
    if LSE is None:
        LSE = torch.empty((shape.B, shape.H, shape.L), dtype=torch.float32, device=Q.device)
    st = lib().bsa_dense_attn_fwd(C.byref(shape.c()), _ptr(Q), _ptr(K), _ptr(V), sm_scale, _ptr(O), _ptr(LSE), _stream())
    _check(st, "bsa_dense_attn_fwd")
    return O, LSE


def dense_attn_bwd(shape: Shape, Q, K, V, O, LSE, dO, sm_scale: Optional[float] = None,
                   dQ=None, dK=None, dV=None, workspace=None):
    if sm_scale is None:
        sm_scale = 1.0 / sqrt(shape.d)
    dQ = torch.empty_like(Q) if dQ is None else dQ
    dK = torch.empty_like(K) if dK is None else dK
    dV = torch.empty_like(V) if dV is None else dV
    if workspace is None:
        workspace = torch.empty(max(1, dense_bwd_workspace_bytes(shape)), dtype=torch.uint8, device=Q.device)
    st = lib().bsa_dense_attn_bwd(C.byref(shape.c()), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(dO),
                                  sm_scale, _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(workspace), workspace.numel(), _stream())
    _check(st, "bsa_dense_attn_bwd")
    return dQ, dK, dV


# ---- the operators around the attention ----------------------------------------------------------
# Their tensors may have any strides that the header allows, so each is checked here for what a pointer cannot tell.
ROPE_PAIRS, ROPE_HALVES = 0, 1


@dataclass(frozen=True)
class Rope:
    """Channels rotated by the grid's t, h and w coordinate, and how they pair up."""
    dt: int
    dh: int
    dw: int
    style: int = ROPE_PAIRS

    def c(self) -> RopeStruct:
        return RopeStruct(self.dt, self.dh, self.dw, self.style)


@dataclass(frozen=True)
class CrossShape:
    B: int
    H: int
    Hkv: int
    Lq: int
    S: int
    d: int
    dtype: int  # F32 or BF16

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == F32 else torch.bfloat16

    def c(self, Q=None, K=None, V=None, O=None) -> CrossStruct:
        """With the strides of the given [B, heads, tokens, d] tensors (contiguous ones where there is none)."""
        d, own = self.d, []
        for t, h, n in ((Q, self.H, self.Lq), (K, self.Hkv, self.S), (V, self.Hkv, self.S), (O, self.H, self.Lq)):
            own += (h * n * d, d, n * d) if t is None else _strides(t)
        return CrossStruct.from_buffer_copy(_CROSS.pack(self.B, self.H, self.Hkv, self.Lq, self.S, d, self.dtype, *own))


def _strides(t: torch.Tensor):
    """Batch, tokens and heads of a [B, heads, tokens, d] tensor."""
    b, h, l, _ = t.stride()  # noqa: E741
    return b, l, h


def _device(t: torch.Tensor) -> torch.device:
    """The device of a call: it has to be the current one, whose stream the work goes to."""
    device = t.device
    if device.type != "cuda" or device.index != torch.cuda.current_device():
        raise ValueError(f"tensors must be on the current GPU, not on {device}")
    return device


# The current stream's handle without the object around it: 0.1 us instead of 2.6, of a call that takes 10.  No public name, so a torch
# without it is served by the public one.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(device: torch.device) -> int:
    """Its current stream."""
    return _raw_stream(device.index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _take(t: Optional[torch.Tensor], name: str, size, dtype, device, dense: bool = False) -> Optional[int]:
    """The address of a tensor of that size, type and device, its last dimension (dense: all of it) contiguous; None for None."""
    if t is None:
        return None
    if t.shape != size or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} must be {tuple(size)} {dtype} on {device}, not {tuple(t.shape)} {t.dtype} on {t.device}")
    if not t.is_contiguous() and (dense or t.stride(-1) != 1 and t.shape[-1] > 1):
        raise ValueError(f"{name} must be contiguous" if dense else f"{name}: the channels of a head must be adjacent")
    return t.data_ptr()


def _scratch(workspace: Optional[torch.Tensor], nbytes: int, device) -> Optional[torch.Tensor]:
    if workspace is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous and on {device}")
    return workspace


def rope_table(shape: Shape, rope: Rope, theta: float = 10000.0, origin=(0, 0, 0), out: Optional[torch.Tensor] = None,
               device="cuda") -> torch.Tensor:
    """cos and sin of every coordinate and pair; origin: coordinates of the grid's first token."""
    nbytes = lib().bsa_rope_table_bytes(C.byref(shape.c()), C.byref(rope.c()))
    if out is None:
        out = torch.empty(max(1, nbytes // 4), dtype=torch.float32, device=device)
    _device(out)
    if out.dtype != torch.float32 or not out.is_contiguous() or out.numel() * 4 < nbytes:
        raise ValueError(f"table must be {nbytes // 4} contiguous floats")
    _check(lib().bsa_rope_table(C.byref(shape.c()), C.byref(rope.c()), theta, *origin, out.data_ptr(), _stream()), "bsa_rope_table")
    return out


def _rope_table_ptr(shape, rope, table: Optional[torch.Tensor], device) -> Optional[int]:
    """shape, rope: the C structures' references."""
    if rope is None or table is None or table.numel() == 0:
        return None
    need = lib().bsa_rope_table_bytes(shape, rope) // 4
    if table.dtype != torch.float32 or table.device != device or not table.is_contiguous() or table.numel() < need:
        raise ValueError(f"table must be {need} contiguous floats on {device}")
    return table.data_ptr()


def _same_strides(tensors, names):
    """The common strides of the [B, L, H, d] tensors that are there (an extent of 1 has none)."""
    first = None
    for t in tensors:
        if t is None:
            continue
        strides = t.stride()
        if first is None:
            first, size = strides, t.shape
        elif strides != first and any(a != b and n > 1 for a, b, n in zip(strides, first, size)):
            raise ValueError(f"{names} must have the same strides")
    return C.byref(StridesStruct(*first[:3]))


def qk_norm_rope_fwd(shape: Shape, rope: Optional[Rope], table: Optional[torch.Tensor], Xq=None, Xk=None, Xv=None,
                     wq=None, wk=None, eps: float = 1e-6, Q=None, K=None, V=None):
    """Xq, Xk, Xv: [B, L, H, d] of the same strides, None to leave one out.  Returns Q, K, V, [B, H, L, d] in the shape's order."""
    X = (Xq, Xk, Xv)
    if all(t is None for t in X):
        raise ValueError("Xq, Xk or Xv must be given")
    dev, dt = _device(next(t for t in X if t is not None)), shape.torch_dtype
    size_in, size_out = (shape.B, shape.L, shape.H, shape.d), (shape.B, shape.H, shape.L, shape.d)
    Y = [torch.empty(size_out, dtype=dt, device=dev) if x is not None and y is None else y for x, y in zip(X, (Q, K, V))]
    args = [_take(x, n, size_in, dt, dev) for x, n in zip(X, ("Xq", "Xk", "Xv"))]
    w = [_take(t, n, (shape.d,), torch.float32, dev, True) for t, n in ((wq, "wq"), (wk, "wk"))]
    outs = [_take(y, n, size_out, dt, dev, True) for y, n in zip(Y, "QKV")]
    sp, rp = C.byref(shape.c()), C.byref(rope.c()) if rope is not None else None
    st = lib().bsa_qk_norm_rope_fwd(sp, rp, _rope_table_ptr(sp, rp, table, dev), *args,
                                    _same_strides(X, "Xq, Xk and Xv"), *w, eps, *outs, _stream_of(dev))
    _check(st, "bsa_qk_norm_rope_fwd")
    return tuple(Y)


def qk_norm_rope_bwd_workspace_bytes(shape: Shape) -> int:
    return lib().bsa_qk_norm_rope_bwd_workspace_bytes(C.byref(shape.c()))


def qk_norm_rope_bwd(shape: Shape, rope: Optional[Rope], table: Optional[torch.Tensor], Xq=None, Xk=None, dQ=None, dK=None, dV=None,
                     wq=None, wk=None, eps: float = 1e-6, dXq=None, dXk=None, dXv=None, dwq=None, dwk=None,
                     workspace: Optional[torch.Tensor] = None, weight_grads: bool = True):
    """Returns dXq, dXk, dXv ([B, L, H, d], contiguous where not given, then all of the same strides), dwq, dwk ([d] float).
    weight_grads=False: dwq and dwk only into memory that is given (None otherwise), and without either one launch less."""
    dY, X = (dQ, dK, dV), (Xq, Xk)
    if all(t is None for t in dY):
        raise ValueError("dQ, dK or dV must be given")
    dev, dt = _device(next(t for t in dY if t is not None)), shape.torch_dtype
    size_x, size_y = (shape.B, shape.L, shape.H, shape.d), (shape.B, shape.H, shape.L, shape.d)
    dX = [torch.empty(size_x, dtype=dt, device=dev) if y is not None and x is None else x for y, x in zip(dY, (dXq, dXk, dXv))]
    dw = [torch.empty(shape.d, dtype=torch.float32, device=dev) if weight_grads and y is not None and t is None else t
          for y, t in zip(dY, (dwq, dwk))]
    xs = [_take(t, n, size_x, dt, dev) for t, n in zip(X, ("Xq", "Xk"))]
    w = [_take(t, n, (shape.d,), torch.float32, dev, True) for t, n in ((wq, "wq"), (wk, "wk"))]
    ys = [_take(t, n, size_y, dt, dev, True) for t, n in zip(dY, ("dQ", "dK", "dV"))]
    outs = [_take(t, n, size_x, dt, dev) for t, n in zip(dX, ("dXq", "dXk", "dXv"))]
    dws = [_take(t, n, (shape.d,), torch.float32, dev, True) for t, n in zip(dw, ("dwq", "dwk"))]
    sp, rp = C.byref(shape.c()), C.byref(rope.c()) if rope is not None else None
    workspace = _scratch(workspace, lib().bsa_qk_norm_rope_bwd_workspace_bytes(sp), dev)
    st = lib().bsa_qk_norm_rope_bwd(sp, rp, _rope_table_ptr(sp, rp, table, dev), *xs,
                                    _same_strides(X, "Xq and Xk") if any(t is not None for t in X) else None, *w, eps, *ys, *outs,
                                    _same_strides(dX, "dXq, dXk and dXv"), *dws, _ptr(workspace),
                                    workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream_of(dev))
    _check(st, "bsa_qk_norm_rope_bwd")
    return (*dX, *dw)


def _like(t: torch.Tensor) -> torch.Tensor:
    """Memory for a tensor like t, in t's order of dimensions, without its repetitions."""
    return torch.empty_like(t) if all(s > 0 for s, n in zip(t.stride(), t.shape) if n > 1) else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def cross_fwd_workspace_bytes(shape: CrossShape) -> int:
    return lib().bsa_cross_attn_fwd_workspace_bytes(C.byref(shape.c()))


def cross_bwd_workspace_bytes(shape: CrossShape) -> int:
    return lib().bsa_cross_attn_bwd_workspace_bytes(C.byref(shape.c()))


def cross_attn_fwd(shape: CrossShape, Q, K, V, kv_len: Optional[torch.Tensor] = None, kv_mask: Optional[torch.Tensor] = None,
                   sm_scale: Optional[float] = None, O=None, LSE=None, workspace: Optional[torch.Tensor] = None):
    """Q: [B, H, Lq, d]; K, V: [B, Hkv, S, d]; any strides with adjacent channels.  kv_len: [B] int32; kv_mask: [B, S] uint8 or bool."""
    dev, dt = _device(Q), shape.torch_dtype
    O = _like(Q) if O is None else O
    LSE = torch.empty((shape.B, shape.H, shape.Lq), dtype=torch.float32, device=dev) if LSE is None else LSE
    qs, ks = (shape.B, shape.H, shape.Lq, shape.d), (shape.B, shape.Hkv, shape.S, shape.d)
    ins = [_take(t, n, s, dt, dev) for t, n, s in ((Q, "Q", qs), (K, "K", ks), (V, "V", ks))]
    valid = _valid(shape, kv_len, kv_mask, dev)
    outs = [_take(O, "O", qs, dt, dev), _take(LSE, "LSE", qs[:3], torch.float32, dev, True)]
    c = shape.c(Q, K, V, O)
    workspace = _scratch(workspace, lib().bsa_cross_attn_fwd_workspace_bytes(C.byref(c)), dev)
    st = lib().bsa_cross_attn_fwd(C.byref(c), *ins, *valid, 1.0 / sqrt(shape.d) if sm_scale is None else sm_scale, *outs, _ptr(workspace),
                                  workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream_of(dev))
    _check(st, "bsa_cross_attn_fwd")
    return O, LSE


def _valid(shape: CrossShape, kv_len, kv_mask, dev):
    if kv_mask is not None and kv_mask.dtype == torch.bool:
        kv_mask = kv_mask.view(torch.uint8)
    return (_take(kv_len, "kv_len", (shape.B,), torch.int32, dev, True),
            _take(kv_mask, "kv_mask", (shape.B, shape.S), torch.uint8, dev, True))


def cross_attn_bwd(shape: CrossShape, Q, K, V, O, LSE, dO, kv_len: Optional[torch.Tensor] = None, kv_mask: Optional[torch.Tensor] = None,
                   sm_scale: Optional[float] = None, dQ=None, dK=None, dV=None, workspace: Optional[torch.Tensor] = None):
    """O, LSE: cross_attn_fwd's for the same arguments, and no others.  dO, dQ, dK, dV may have strides of their own.  Of K and V that
    repeat (expanded), dK and dV hold every repetition's gradient."""
    dev, dt = _device(Q), shape.torch_dtype
    dQ, dK, dV = (_like(t) if g is None else g for t, g in ((Q, dQ), (K, dK), (V, dV)))
    qs, ks = (shape.B, shape.H, shape.Lq, shape.d), (shape.B, shape.Hkv, shape.S, shape.d)
    ins = [_take(t, n, s, dt, dev) for t, n, s in ((Q, "Q", qs), (K, "K", ks), (V, "V", ks), (O, "O", qs))]
    ins += [_take(LSE, "LSE", qs[:3], torch.float32, dev, True), _take(dO, "dO", qs, dt, dev)]
    valid = _valid(shape, kv_len, kv_mask, dev)
    outs = [_take(t, n, s, dt, dev) for t, n, s in ((dQ, "dQ", qs), (dK, "dK", ks), (dV, "dV", ks))]
    c = shape.c(Q, K, V, O)
    grads = _FOUR_STRIDES.from_buffer_copy(_FOUR.pack(*_strides(dO), *_strides(dQ), *_strides(dK), *_strides(dV)))
    workspace = _scratch(workspace, lib().bsa_cross_attn_bwd_workspace_bytes(C.byref(c)), dev)
    st = lib().bsa_cross_attn_bwd(C.byref(c), *ins, *valid, 1.0 / sqrt(shape.d) if sm_scale is None else sm_scale, *outs, grads,
                                  _ptr(workspace), workspace.numel() * workspace.element_size() if workspace is not None else 0, _stream_of(dev))
    _check(st, "bsa_cross_attn_bwd")
    return dQ, dK, dV


def mfma_probe(workgroups: int, iters: int, sink=None) -> int:
    """Enqueue the register-resident matrix-core loop; returns the flops the launch performs."""
    if sink is None:
        sink = torch.empty(workgroups * 256, dtype=torch.float32, device="cuda")
    if sink.numel() < workgroups * 256:
        raise ValueError("sink too small")
    flops = lib().bsa_mfma_probe(workgroups, iters, _ptr(sink), _stream())
    if flops < 0:
        _check(int(flops), "bsa_mfma_probe")
    return int(flops)
