"""GB300-native BF16 component-product GEMM emulation (arXiv 2609.04663).

Thin ctypes binding over the C-ABI of ``include/emu.h`` and
``include/emu_experts.h`` (library ``_emu.so`` built in-tree by
``_build.py``).  The functions named ``emu_*`` take plain integers (device
pointers, sizes, the raw CUDA stream handle) and return the ``emu_status``
code, exactly as the C entry points do.  The
tensor-level helpers below them only allocate device memory with PyTorch and
marshal pointers: every step of the method runs in the CUDA kernels.

There is no CPU fallback: importing this package without the compiled
library raises.
"""
from __future__ import annotations

import collections
import ctypes
import os

from . import _build

_lib = None

EMU_OK = 0
STATUS = {0: "ok", 1: "invalid argument", 2: "misaligned", 3: "workspace too small", 4: "CUDA error",
          5: "unsupported size"}
FLAG_NONFINITE, FLAG_RANGE, FLAG_SLICE, FLAG_TIMEOUT, FLAG_INDEX = 0x1, 0x2, 0x4, 0x8, 0x10
OP_N, OP_T = 0, 1
F32, BF16 = 0, 1
KEEP_FLAGS = 0x100
ZERO_LEVEL = -(2 ** 31)

_SIGS = {
    # name: (restype, argtypes)
    "emu_split_workspace_bytes": ("size", ["i"]),
    "emu_split_f32": ("i", ["p", "l", "l", "l", "i", "p", "l", "p", "size", "p"]),
    "emu_split_f64": ("i", ["p", "l", "l", "l", "i", "p", "l", "p", "p", "size", "p"]),
    "emu_split_f64_slices": ("i", ["p", "l", "l", "l", "i", "p", "l", "i", "p", "p", "size", "p"]),
    "emu_gemm_workspace_bytes": ("size", ["i", "l", "l", "l"]),
    "emu_split_f32_pair": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "p", "l", "p", "size", "p"]),
    "emu_split_f64_pair": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "p", "l", "i", "p", "p", "p", "size", "p"]),
    "emu_gemm_f32": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "l", "p", "size", "p"]),
    "emu_gemm_f64": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "l", "i", "p", "size", "p"]),
    "emu_gemm_f32_fused": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "l", "p", "size", "p"]),
    "emu_gemm_f64_merged_workspace_bytes": ("size", ["l", "l", "l"]),
    "emu_gemm_f64_merged": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "l", "i", "i", "p", "size", "p"]),
    "emu_prodsum_f32": ("i", ["l", "l", "l", "p", "p", "l", "p", "l", "p", "size", "p"]),
    "emu_prodsum_f64": ("i", ["l", "l", "l", "p", "p", "l", "p", "p", "i", "p", "l", "p", "size", "p"]),
    "emu_gemm_f64_noalloc": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "l", "i", "p", "p"]),
    "emu_gemm_host_workspace_bytes": ("size", ["i", "l", "l", "l"]),
    "emu_gemm_ex_workspace_bytes": ("size", ["i", "l", "l", "l"]),
    "emu_prodsum_workspace_bytes": ("size", ["i", "l", "l"]),
    "emu_prodsum_f64_tile_columns": ("i", ["l", "l"]),
    "emu_prodsum_f64_tile_rows": ("i", ["l", "l"]),
    "emu_prodsum_f64_launches": ("i", ["l", "l"]),
    "emu_prodsum_f32_launches": ("i", ["l", "l"]),
    "emu_prodsum_f32_tile_columns": ("i", ["l", "l"]),
    "emu_prodsum_f32_tile_rows": ("i", ["l", "l"]),
    "emu_split_f64_rowcol_workspace_bytes": ("size", ["l"]),
    "emu_split_f64_rowcol": ("i", ["p", "l", "l", "l", "i", "p", "l", "p", "p", "size", "p"]),
    "emu_gemm_f64_rowcol_workspace_bytes": ("size", ["l", "l", "l"]),
    "emu_gemm_f64_rowcol": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "l", "i", "p", "size", "p"]),
    "emu_gemm_ex_f32": ("i", ["i", "i", "l", "l", "l", "f", "p", "l", "p", "l", "f", "p", "l", "p", "size", "p"]),
    "emu_gemm_ex_f64": ("i", ["i", "i", "l", "l", "l", "d", "p", "l", "p", "l", "d", "p", "l", "i", "p", "size", "p"]),
    "emu_gemm_f32_host": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "l", "p", "size", "p"]),
    "emu_gemm_f64_host": ("i", ["l", "l", "l", "p", "l", "p", "l", "p", "l", "i", "p", "size", "p"]),
    "emu_grouped_plane_rows": ("l", ["l", "l"]),
    "emu_grouped_split": ("i", ["i", "l", "l", "l", "p", "l", "l", "p", "l", "p", "size", "p"]),
    "emu_grouped_split_rows": ("i", ["i", "l", "l", "p", "l", "l", "p", "p", "l", "p", "l", "p", "size", "p"]),
    "emu_grouped_prodsum": ("i", ["i", "i", "l", "l", "l", "l", "p", "l", "i", "p", "l", "l", "p", "p", "i", "l", "p",
                                  "size", "p"]),
    "emu_grouped_gemm_workspace_bytes": ("size", ["i", "l", "l", "l", "l"]),
    "emu_grouped_gemm_f32": ("i", ["i", "l", "l", "l", "l", "p", "l", "l", "p", "p", "l", "l", "p", "p", "l", "p",
                                   "size", "p"]),
    "emu_grouped_prodsum_wgrad": ("i", ["i", "l", "l", "l", "l", "p", "l", "i", "p", "l", "i", "p", "p", "i", "l", "l",
                                        "p", "size", "p"]),
    "emu_w4_workspace_bytes": ("size", ["i", "l", "l"]),
    "emu_w4_matvec": ("i", ["i", "l", "l", "l", "l", "l", "p", "l", "p", "p", "i", "p", "p", "p", "l", "p", "size",
                            "p"]),
    "emu_route_workspace_bytes": ("size", ["l", "l", "l"]),
    "emu_route": ("i", ["i", "l", "l", "l", "i", "p", "l", "p", "p", "p", "p", "p", "p", "size", "p"]),
    "emu_selftest_route_timeout": ("i", ["u32", "l", "l", "l", "p", "l", "p", "p", "p", "p", "p", "p", "size", "p"]),
    "emu_route_backward": ("i", ["i", "l", "l", "l", "i", "p", "l", "p", "p", "p", "l", "p"]),
    "emu_rows_combine": ("i", ["i", "l", "l", "l", "p", "l", "l", "p", "p", "p", "l", "p"]),
    "emu_rows_combine_backward": ("i", ["i", "l", "l", "l", "p", "l", "p", "l", "l", "p", "p", "p", "l", "p", "p"]),
    "emu_rows_combine_workspace_bytes": ("size", ["l"]),
    "emu_rows_combine_backward_full": ("i", ["i", "l", "l", "l", "p", "l", "p", "l", "l", "p", "p", "p", "l", "p", "p",
                                             "size", "p"]),
    "emu_read_flags": ("i", ["p", "p", "p"]),
    "emu_selftest_timeout": ("i", ["p", "size", "u32", "p"]),
    "emu_status_string": ("str", ["i"]),
}
_CT = {"i": ctypes.c_int, "l": ctypes.c_int64, "p": ctypes.c_void_p, "size": ctypes.c_size_t,
       "u32": ctypes.c_uint32, "str": ctypes.c_char_p, "f": ctypes.c_float, "d": ctypes.c_double}


class EmuError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {STATUS.get(status, status)} (status {status})")
        self.status = status


def library_path() -> str:
    return _build.SO


def load():
    """Load ``_emu.so`` (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_build.SO):
            raise ImportError(f"CUDA emulation library not built: {_build.SO} is missing "
                              "(run paper_2609_04663_gb300._build.build())")
        lib = ctypes.CDLL(_build.SO)
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype = _CT[res]
            fn.argtypes = [_CT[a] for a in args]
        _lib = lib
    return _lib


def _mk(name):
    def f(*args):
        return getattr(load(), name)(*args)
    f.__name__ = name
    f.__doc__ = f"C-ABI ``{name}`` (declared under include/); returns its result unchanged."
    return f


emu_split_workspace_bytes = _mk("emu_split_workspace_bytes")
emu_split_f32 = _mk("emu_split_f32")
emu_split_f64 = _mk("emu_split_f64")
emu_split_f64_slices = _mk("emu_split_f64_slices")
emu_gemm_workspace_bytes = _mk("emu_gemm_workspace_bytes")
emu_split_f32_pair = _mk("emu_split_f32_pair")
emu_split_f64_pair = _mk("emu_split_f64_pair")
emu_gemm_f32 = _mk("emu_gemm_f32")
emu_gemm_f64 = _mk("emu_gemm_f64")
emu_gemm_f32_fused = _mk("emu_gemm_f32_fused")
emu_gemm_f64_merged_workspace_bytes = _mk("emu_gemm_f64_merged_workspace_bytes")
emu_gemm_f64_merged = _mk("emu_gemm_f64_merged")
emu_prodsum_f32 = _mk("emu_prodsum_f32")
emu_prodsum_f64 = _mk("emu_prodsum_f64")
emu_gemm_f64_noalloc = _mk("emu_gemm_f64_noalloc")
emu_gemm_host_workspace_bytes = _mk("emu_gemm_host_workspace_bytes")
emu_gemm_ex_workspace_bytes = _mk("emu_gemm_ex_workspace_bytes")
emu_prodsum_workspace_bytes = _mk("emu_prodsum_workspace_bytes")
emu_prodsum_f64_tile_columns = _mk("emu_prodsum_f64_tile_columns")
emu_prodsum_f64_tile_rows = _mk("emu_prodsum_f64_tile_rows")
emu_prodsum_f64_launches = _mk("emu_prodsum_f64_launches")
emu_prodsum_f32_launches = _mk("emu_prodsum_f32_launches")
emu_prodsum_f32_tile_columns = _mk("emu_prodsum_f32_tile_columns")
emu_prodsum_f32_tile_rows = _mk("emu_prodsum_f32_tile_rows")
emu_split_f64_rowcol_workspace_bytes = _mk("emu_split_f64_rowcol_workspace_bytes")
emu_split_f64_rowcol = _mk("emu_split_f64_rowcol")
emu_gemm_f64_rowcol_workspace_bytes = _mk("emu_gemm_f64_rowcol_workspace_bytes")
emu_gemm_f64_rowcol = _mk("emu_gemm_f64_rowcol")
emu_gemm_ex_f32 = _mk("emu_gemm_ex_f32")
emu_gemm_ex_f64 = _mk("emu_gemm_ex_f64")
emu_gemm_f32_host = _mk("emu_gemm_f32_host")
emu_gemm_f64_host = _mk("emu_gemm_f64_host")
emu_grouped_plane_rows = _mk("emu_grouped_plane_rows")
emu_grouped_split = _mk("emu_grouped_split")
emu_grouped_split_rows = _mk("emu_grouped_split_rows")
emu_grouped_prodsum = _mk("emu_grouped_prodsum")
emu_grouped_gemm_workspace_bytes = _mk("emu_grouped_gemm_workspace_bytes")
emu_grouped_gemm_f32 = _mk("emu_grouped_gemm_f32")
emu_grouped_prodsum_wgrad = _mk("emu_grouped_prodsum_wgrad")
emu_w4_workspace_bytes = _mk("emu_w4_workspace_bytes")
emu_w4_matvec = _mk("emu_w4_matvec")
emu_route_workspace_bytes = _mk("emu_route_workspace_bytes")
emu_route = _mk("emu_route")
emu_selftest_route_timeout = _mk("emu_selftest_route_timeout")
emu_route_backward = _mk("emu_route_backward")
emu_rows_combine = _mk("emu_rows_combine")
emu_rows_combine_backward = _mk("emu_rows_combine_backward")
emu_rows_combine_workspace_bytes = _mk("emu_rows_combine_workspace_bytes")
emu_rows_combine_backward_full = _mk("emu_rows_combine_backward_full")
emu_read_flags = _mk("emu_read_flags")
emu_selftest_timeout = _mk("emu_selftest_timeout")
emu_status_string = _mk("emu_status_string")


# ------------------------------------------------------------ tensor helpers
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _stream(stream):
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream if hasattr(s, "cuda_stream") else int(s)


def _check(status, where):
    if status != EMU_OK:
        raise EmuError(status, where)


def workspace(nbytes: int, device="cuda"):
    """A device workspace (uint8 tensor) of at least nbytes, 256-byte aligned by the allocator."""
    torch = _torch()
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


def read_flags(ws, stream=None) -> int:
    out = ctypes.c_uint32(0)
    _check(emu_read_flags(ws.data_ptr(), ctypes.addressof(out), _stream(stream)), "emu_read_flags")
    return int(out.value)


def gemm_ldk(K: int) -> int:
    """Leading dimension of the K-major planes inside a GEMM workspace."""
    return (max(K, 1) + 7) // 8 * 8


def split_f32(X, transpose: bool = False, ldcomp: int | None = None, ws=None, stream=None):
    """Eq. (fp32split) on the GPU: returns (planes int16 [3, rows_out, ldcomp], ws)."""
    torch = _torch()
    rows, cols = X.shape
    rows_out, cols_out = (cols, rows) if transpose else (rows, cols)
    ldcomp = ldcomp or cols_out
    planes = torch.zeros((3, rows_out, ldcomp), dtype=torch.int16, device=X.device)
    ws = ws if ws is not None else workspace(emu_split_workspace_bytes(32), X.device)
    _check(emu_split_f32(X.data_ptr(), rows, cols, X.stride(0), int(transpose), planes.data_ptr(), ldcomp,
                         ws.data_ptr(), ws.numel(), _stream(stream)), "emu_split_f32")
    return planes, ws


def split_f64(X, transpose: bool = False, ldcomp: int | None = None, ws=None, stream=None, nslices: int = 6):
    """Eq. (fp64split) on the GPU: returns (planes int16 [6, rows_out, ldcomp], v int32[6] (device), ws).
    nslices < 6 calls emu_split_f64_slices (planes and levels from nslices on unspecified)."""
    torch = _torch()
    rows, cols = X.shape
    rows_out, cols_out = (cols, rows) if transpose else (rows, cols)
    ldcomp = ldcomp or cols_out
    planes = torch.zeros((6, rows_out, ldcomp), dtype=torch.int16, device=X.device)
    v = torch.empty(6, dtype=torch.int32, device=X.device)
    ws = ws if ws is not None else workspace(emu_split_workspace_bytes(64), X.device)
    if nslices == 6:
        _check(emu_split_f64(X.data_ptr(), rows, cols, X.stride(0), int(transpose), planes.data_ptr(), ldcomp,
                             v.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream)), "emu_split_f64")
    else:
        _check(emu_split_f64_slices(X.data_ptr(), rows, cols, X.stride(0), int(transpose), planes.data_ptr(), ldcomp,
                                    int(nslices), v.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream)),
               "emu_split_f64_slices")
    return planes, v, ws


def split_f64_rowcol(X, transpose: bool = False, ldcomp: int | None = None, ws=None, stream=None):
    """emu_split_f64_rowcol: levels per row of X (per column when transposed).
    Returns (planes int16 [6, plane_rows, ldcomp], v int32 [6, plane_rows] (device), ws)."""
    torch = _torch()
    rows, cols = X.shape
    prow, pcols = (cols, rows) if transpose else (rows, cols)
    ldcomp = ldcomp or pcols
    planes = torch.zeros((6, prow, ldcomp), dtype=torch.int16, device=X.device)
    v = torch.empty((6, prow), dtype=torch.int32, device=X.device)
    ws = ws if ws is not None else workspace(emu_split_f64_rowcol_workspace_bytes(prow), X.device)
    _check(emu_split_f64_rowcol(X.data_ptr(), rows, cols, X.stride(0), int(transpose), planes.data_ptr(), ldcomp,
                                v.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream)), "emu_split_f64_rowcol")
    return planes, v, ws


def gemm_f64_rowcol(A, B, nprod: int, C=None, ws=None, stream=None):
    """emu_gemm_f64_rowcol: Algorithm 2 with levels per row of A and per column of B."""
    torch = _torch()
    M, K = A.shape
    N = B.shape[1]
    C = C if C is not None else torch.empty((M, N), dtype=torch.float64, device=A.device)
    ws = ws if ws is not None else workspace(emu_gemm_f64_rowcol_workspace_bytes(M, N, K), A.device)
    _check(emu_gemm_f64_rowcol(M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C.data_ptr(),
                               C.stride(0), int(nprod), ws.data_ptr(), ws.numel(), _stream(stream)),
           "emu_gemm_f64_rowcol")
    return C, ws


def gemm_f32(A, B, C=None, ws=None, stream=None):
    """Algorithm 1 on the GPU: C = A.B for FP32 row-major A (M x K), B (K x N)."""
    torch = _torch()
    M, K = A.shape
    N = B.shape[1]
    C = C if C is not None else torch.empty((M, N), dtype=torch.float32, device=A.device)
    ws = ws if ws is not None else workspace(emu_gemm_workspace_bytes(32, M, N, K), A.device)
    _check(emu_gemm_f32(M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C.data_ptr(), C.stride(0),
                        ws.data_ptr(), ws.numel(), _stream(stream)), "emu_gemm_f32")
    return C, ws


def gemm_f32_fused(A, B, C=None, ws=None, stream=None):
    """emu_gemm_f32_fused: Algorithm 1 with the split inside the product-sum
    (no planes in memory); C bit-identical to gemm_f32."""
    torch = _torch()
    M, K = A.shape
    N = B.shape[1]
    C = C if C is not None else torch.empty((M, N), dtype=torch.float32, device=A.device)
    ws = ws if ws is not None else workspace(emu_split_workspace_bytes(32), A.device)
    _check(emu_gemm_f32_fused(M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C.data_ptr(),
                              C.stride(0), ws.data_ptr(), ws.numel(), _stream(stream)), "emu_gemm_f32_fused")
    return C, ws


def gemm_f64(A, B, nprod: int, C=None, ws=None, stream=None):
    """Algorithm 2 on the GPU: C = A.B for FP64 A, B with nprod in {6, 10, 15, 21}."""
    torch = _torch()
    M, K = A.shape
    N = B.shape[1]
    C = C if C is not None else torch.empty((M, N), dtype=torch.float64, device=A.device)
    ws = ws if ws is not None else workspace(emu_gemm_workspace_bytes(64, M, N, K), A.device)
    _check(emu_gemm_f64(M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C.data_ptr(), C.stride(0),
                        int(nprod), ws.data_ptr(), ws.numel(), _stream(stream)), "emu_gemm_f64")
    return C, ws


def gemm_f64_merged(A, B, nprod: int, merge_from: int, C=None, ws=None, stream=None):
    """emu_gemm_f64_merged: Algorithm 2's head (i + j < merge_from) plus the
    remaining products of S_d accumulated in one FP32 tail, added last."""
    torch = _torch()
    M, K = A.shape
    N = B.shape[1]
    C = C if C is not None else torch.empty((M, N), dtype=torch.float64, device=A.device)
    ws = ws if ws is not None else workspace(emu_gemm_f64_merged_workspace_bytes(M, N, K), A.device)
    _check(emu_gemm_f64_merged(M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C.data_ptr(),
                               C.stride(0), int(nprod), int(merge_from), ws.data_ptr(), ws.numel(), _stream(stream)),
           "emu_gemm_f64_merged")
    return C, ws


def gemm_ex(A, B, opA: int = OP_N, opB: int = OP_N, alpha: float = 1.0, beta: float = 0.0, C=None,
            nprod: int | None = None, ws=None, stream=None):
    """emu_gemm_ex_*: C <- alpha op(A) op(B) + beta C for device tensors A, B
    as stored (op = OP_T reads the stored matrix transposed).  FP32 tensors
    run Algorithm 1, FP64 tensors Algorithm 2 with nprod products."""
    torch = _torch()
    M, K = (A.shape[1], A.shape[0]) if opA == OP_T else (A.shape[0], A.shape[1])
    N = B.shape[0] if opB == OP_T else B.shape[1]
    f64 = A.dtype == torch.float64
    C = C if C is not None else torch.zeros((M, N), dtype=A.dtype, device=A.device)
    ws = ws if ws is not None else workspace(emu_gemm_ex_workspace_bytes(64 if f64 else 32, M, N, K), A.device)
    if f64:
        r = emu_gemm_ex_f64(opA, opB, M, N, K, float(alpha), A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0),
                            float(beta), C.data_ptr(), C.stride(0), int(nprod), ws.data_ptr(), ws.numel(),
                            _stream(stream))
    else:
        r = emu_gemm_ex_f32(opA, opB, M, N, K, float(alpha), A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0),
                            float(beta), C.data_ptr(), C.stride(0), ws.data_ptr(), ws.numel(), _stream(stream))
    _check(r, "emu_gemm_ex_f64" if f64 else "emu_gemm_ex_f32")
    return C, ws


def gemm_host(A, B, nprod: int | None = None, C=None, ws=None, stream=None, device="cuda"):
    """emu_gemm_f32_host / emu_gemm_f64_host: C = A.B with A, B, C in host
    memory (CPU tensors; pinned ones give asynchronous full-speed copies).
    FP32 inputs run Algorithm 1, FP64 inputs Algorithm 2 with nprod products.
    Returns (C, ws) after enqueueing; synchronise the stream before reading C."""
    torch = _torch()
    M, K = A.shape
    N = B.shape[1]
    f64 = A.dtype == torch.float64
    C = C if C is not None else torch.empty((M, N), dtype=A.dtype, pin_memory=True)
    mode = 64 if f64 else 32
    ws = ws if ws is not None else workspace(emu_gemm_host_workspace_bytes(mode, M, N, K), device)
    if f64:
        r = emu_gemm_f64_host(M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C.data_ptr(),
                              C.stride(0), int(nprod), ws.data_ptr(), ws.numel(), _stream(stream))
    else:
        r = emu_gemm_f32_host(M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C.data_ptr(),
                              C.stride(0), ws.data_ptr(), ws.numel(), _stream(stream))
    _check(r, "emu_gemm_f64_host" if f64 else "emu_gemm_f32_host")
    return C, ws


def prodsum_f32(Ap, Bp, M: int, N: int, K: int, C=None, ws=None, stream=None):
    """Product-sum alone from planes Ap [3, M, ldcomp], Bp [3, N, ldcomp] (K-major)."""
    torch = _torch()
    C = C if C is not None else torch.empty((M, N), dtype=torch.float32, device=Ap.device)
    ws = ws if ws is not None else workspace(emu_split_workspace_bytes(32), Ap.device)
    _check(emu_prodsum_f32(M, N, K, Ap.data_ptr(), Bp.data_ptr(), Ap.shape[2], C.data_ptr(), C.stride(0),
                           ws.data_ptr(), ws.numel(), _stream(stream)), "emu_prodsum_f32")
    return C, ws


def prodsum_f64(Ap, Bp, M: int, N: int, K: int, nprod: int, vA=None, vB=None, C=None, ws=None, stream=None):
    """FP64-mode product-sum alone from planes Ap [6, M, ldcomp], Bp [6, N, ldcomp];
    vA, vB: the level exponents emu_split_f64 returned for A and B (or None)."""
    torch = _torch()
    C = C if C is not None else torch.empty((M, N), dtype=torch.float64, device=Ap.device)
    ws = ws if ws is not None else workspace(emu_prodsum_workspace_bytes(64, M, N), Ap.device)
    _check(emu_prodsum_f64(M, N, K, Ap.data_ptr(), Bp.data_ptr(), Ap.shape[2],
                           vA.data_ptr() if vA is not None else None, vB.data_ptr() if vB is not None else None,
                           int(nprod), C.data_ptr(), C.stride(0), ws.data_ptr(), ws.numel(), _stream(stream)),
           "emu_prodsum_f64")
    return C, ws


# ------------------------------------------------------------- expert layers
# Small calls take a few microseconds on the GPU, so these helpers keep the
# host's share small: plain comparisons, messages only made when one fails.
def _bad(where, what):
    raise ValueError(f"{where}: {what}")


def _raw_stream(stream, device):
    """The CUDA stream handle to launch on (None: PyTorch's current one)."""
    if stream is None:
        return _torch_module._C._cuda_getCurrentRawStream(device.index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _torch_stream(stream, device):
    torch = _torch()
    if stream is None:
        return torch.cuda.current_stream(device)
    return stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device)


def _empty(shape, dtype, device, stream):
    """torch.empty whose memory belongs to the stream that the kernels use."""
    if stream is None:
        return _torch_module.empty(shape, dtype=dtype, device=device)
    with _torch().cuda.stream(_torch_stream(stream, device)):
        return _torch_module.empty(shape, dtype=dtype, device=device)


_codes = {}


def _dtype(t, where):
    """The EMU_* code of a tensor's type (every call asks for one first: loads the library)."""
    code = _codes.get(t.dtype)
    if code is None:
        torch = _torch()
        load()
        _codes.update({torch.float32: F32, torch.bfloat16: BF16})
        code = _codes.get(t.dtype)
        if code is None:
            _bad(where, f"float32 or bfloat16 is needed, got {t.dtype}")
    return code


def _ints(t, numel, device, where):
    """Address of an int32 tensor of `numel` entries (None: any number)."""
    if t.dtype is not _torch_module.int32 or t.device != device or not t.is_contiguous():
        _bad(where, f"a contiguous int32 tensor on {device} is needed")
    if numel is not None and t.numel() != numel:
        _bad(where, f"{numel} entries are needed, got {t.numel()}")
    return t.data_ptr()


def _pitch(t, where, device=None):
    """Row pitch of a CUDA tensor whose rows are contiguous (on `device`, if given)."""
    if not t.is_cuda or (device is not None and t.device != device):
        _bad(where, f"a tensor on {device or 'a GPU'} is needed, got one on {t.device}")
    if t.is_contiguous():
        return t.shape[-1] or 1
    rows, cols = t.shape[-2:]
    st = t.stride()
    if cols > 1 and st[-1] != 1:
        _bad(where, "rows have to be contiguous")
    pitch = st[-2] if rows > 1 else cols
    if pitch < cols:
        _bad(where, "rows overlap")
    return pitch or 1


class GroupedPlanes:
    """BF16 planes of an operand of the products grouped by expert, from
    grouped_split: planes int16 [S, plane rows, ld]; `shape` is the operand's
    (rows, cols) for token rows in group order, (G, rows, cols) for weights.
    Token rows are padded for the `ends` that they were split with: a call
    with other ends needs other planes."""

    def __init__(self, planes, shape, padded):
        self.planes, self.shape, self.padded = planes, tuple(shape), padded
        self.device, self.nslices, self.ld = planes.device, planes.shape[0], planes.shape[2]


def _whole_planes(t, G, where):
    """Refuses a plane set that does not have the plane rows of its shape in G groups:
    the kernels take them as given."""
    rows = emu_grouped_plane_rows(t.shape[0], G) if t.padded else G * t.shape[1]
    if t.planes.shape[1] != rows:
        _bad(where, f"a plane set made for {G} groups is needed")


def _slices(t, where):
    return t.nslices if isinstance(t, GroupedPlanes) else (3 if _dtype(t, where) == F32 else 1)


def grouped_split(X, ends=None, src=None, planes=None, ws=None, stream=None):
    """emu_grouped_split / emu_grouped_split_rows: the planes of weights X
    [G, rows, cols] (ends None), or of token rows X[src] (src None: X) grouped
    by ends; three for FP32 (Eq. (fp32split)), one for BF16.  A plane set can
    stand for its operand in grouped_gemm and grouped_wgrad, in all directions.
    Pays for FP32 weights that meet hundreds of rows each; with a few the
    products are faster on the weights themselves (62 rows over 14 experts of
    6528 x 3232, product and both gradients: 1.53 ms with planes, 0.82 without).
    The flags of the call are in ws, where a caller gives one."""
    return _split(X, ends, src, planes, ws, stream, 0)


def _split(X, ends, src, planes, ws, stream, keep):
    """grouped_split; keep: KEEP_FLAGS where ws holds the flags of another operand's split, else 0."""
    torch, where = _torch(), "grouped_split"
    dt, ldx, dev = _dtype(X, where), _pitch(X, where), X.device
    cols = X.shape[-1]
    S, ld = (3 if dt == F32 else 1), gemm_ldk(cols)
    if ws is None:
        ws = _empty(emu_split_workspace_bytes(32), torch.uint8, dev, stream)
    if ends is None:
        if X.dim() != 3 or src is not None:
            _bad(where, "weights are [G, rows, cols]; token rows need ends")
        G, rows = X.shape[0], X.shape[1]
        shape, prows = (G, rows, cols), G * rows
    else:
        if X.dim() != 2:
            _bad(where, "token rows are [rows, cols]")
        G, rows = ends.numel(), (src.numel() if src is not None else X.shape[0])
        shape, prows = (rows, cols), _lib.emu_grouped_plane_rows(rows, G)
    if planes is None:
        planes = _empty((S, prows, ld), torch.int16, dev, stream)
    elif planes.shape != (S, prows, ld) or planes.dtype is not torch.int16 or not planes.is_contiguous():
        _bad(where, f"planes have to be contiguous int16 {(S, prows, ld)}")
    if ends is None:
        r = _lib.emu_grouped_split(dt | keep, G, rows, cols, X.data_ptr(), ldx, X.stride(0) if G > 1 else 0,
                                     planes.data_ptr(), ld, ws.data_ptr(), ws.numel(), _raw_stream(stream, dev))
    else:
        r = _lib.emu_grouped_split_rows(dt | keep, rows, cols, X.data_ptr(), X.shape[0], ldx,
                                          _ints(src, None, dev, "grouped_split: src") if src is not None else None,
                                          _ints(ends, G, dev, "grouped_split: ends"), G, planes.data_ptr(), ld,
                                          ws.data_ptr(), ws.numel(), _raw_stream(stream, dev))
    _check(r, "emu_grouped_split")
    return GroupedPlanes(planes, shape, ends is not None)


def _tma_ok(t, pitch):
    """Whether a BF16 tensor can be read by the tensor memory accelerator as it stands."""
    return (t.data_ptr() % 16 == 0 and pitch % 8 == 0 and
            (t.dim() < 3 or t.shape[0] <= 1 or (t.stride(0) % 8 == 0 and t.stride(0) >= t.shape[1] * pitch)))


def grouped_workspace(X, W, ends, opW: int = OP_N, src=None, train: bool = False):
    """A workspace for grouped_gemm(X, W, ends, opW, src) and, with train, for
    the splits and gradients of the same operands."""
    rows = src.numel() if src is not None else X.shape[0]
    G = ends.numel()
    K, N = (W.shape[2], W.shape[1]) if opW == OP_T else (W.shape[1], W.shape[2])
    dt = F32 if not isinstance(X, GroupedPlanes) and X.dtype == _torch().float32 else BF16
    need = emu_grouped_gemm_workspace_bytes(dt, G, rows, N, K)
    if train:                                         # the rows' gradient: the product with K and N exchanged
        need = max(need, emu_grouped_gemm_workspace_bytes(dt, G, rows, K, N))
    return workspace(need, X.device)


def grouped_gemm(X, W, ends, opW: int = OP_N, src=None, Y=None, ws=None, stream=None):
    """Y[r] = X[src[r]] op(W_g) for the rows r of group g (src None: X[r]);
    W [G, K, N] (OP_N) or [G, N, K] (OP_T).  FP32 operands multiply by six BF16
    products (Algorithm 1), BF16 ones by one; X and W may each be a plane set
    of grouped_split.  Y: FP32, or BF16 / FP32 for BF16 operands (given Y
    decides; BF16 otherwise).  Returns (Y, ws).  The gradient of X is
    grouped_gemm(dY, W, ends, the other op)."""
    torch, where = _torch(), "grouped_gemm"
    G, dev = ends.numel(), X.device
    xp, wp = isinstance(X, GroupedPlanes), isinstance(W, GroupedPlanes)
    if len(W.shape) != 3 or W.shape[0] != G:
        _bad(where, f"W has to be [{G}, ., .], got {tuple(W.shape)}")
    if len(X.shape) != 2 or (xp and (not X.padded or src is not None)):
        _bad(where, "X has to be token rows")
    K, N = (W.shape[2], W.shape[1]) if opW == OP_T else (W.shape[1], W.shape[2])
    if X.shape[1] != K:
        _bad(where, f"X has {X.shape[1]} columns, op(W) {K} rows")
    if xp:
        _whole_planes(X, G, "grouped_gemm: X")
    if wp:
        _whole_planes(W, G, "grouped_gemm: W")
    S = _slices(X, where)
    if S != _slices(W, where) or W.device != dev:
        _bad(where, "X and W have to be of one type, on one device")
    rows = src.numel() if src is not None else X.shape[0]
    if Y is None:
        Y, yt = _empty((rows, N), torch.float32 if S == 3 else torch.bfloat16, dev, stream), (F32 if S == 3 else BF16)
    else:
        yt = _dtype(Y, where)
    ldy = _pitch(Y, "grouped_gemm: Y", dev)
    if Y.shape != (rows, N) or (S == 3 and yt != F32):
        _bad(where, "Y has another shape or type")
    pe = _ints(ends, G, dev, "grouped_gemm: ends")
    ldx = X.ld if xp else _pitch(X, "grouped_gemm: X")
    ldw = W.ld if wp else _pitch(W, "grouped_gemm: W")
    raw = _raw_stream(stream, dev)
    if S == 3 and not xp and not wp:
        ps = _ints(src, None, dev, "grouped_gemm: src") if src is not None else None
        if ws is None:
            ws = _empty(emu_grouped_gemm_workspace_bytes(F32, G, rows, N, K), torch.uint8, dev, stream)
        r = _lib.emu_grouped_gemm_f32(opW, G, rows, N, K, X.data_ptr(), X.shape[0], ldx, ps, W.data_ptr(), ldw,
                                        W.stride(0) if G > 1 else 0, pe, Y.data_ptr(), ldy, ws.data_ptr(), ws.numel(),
                                        raw)
        if r:
            _check(r, "emu_grouped_gemm_f32")
        return Y, ws
    if ws is None:
        ws = _empty(emu_split_workspace_bytes(32), torch.uint8, dev, stream)
    keep = 0                                          # the first launch clears the flag word, the others add to it
    if not xp and (S == 3 or src is not None or not _tma_ok(X, ldx)):
        X, xp, keep = _split(X, ends, src, None, ws, stream, keep), True, KEEP_FLAGS
        ldx = X.ld
    if not wp and (S == 3 or not _tma_ok(W, ldw)):
        W, wp, keep = _split(W, None, None, None, ws, stream, keep), True, KEEP_FLAGS
        ldw = W.ld
    r = _lib.emu_grouped_prodsum(S | keep, opW, G, rows, N, K, X.planes.data_ptr() if xp else X.data_ptr(), ldx, int(xp),
                                   W.planes.data_ptr() if wp else W.data_ptr(), ldw,
                                   W.shape[1] * ldw if wp or G <= 1 else W.stride(0), pe, Y.data_ptr(), yt, ldy,
                                   ws.data_ptr(), ws.numel(), raw)
    if r:
        _check(r, "emu_grouped_prodsum")
    return Y, ws


def _token_operand(t, ends, src, ws, stream, keep, where):
    """(operand, address, row pitch, padded, slices, keep) of token rows: BF16 rows as
    they stand where the tensor memory accelerator can read them, else planes.  keep:
    KEEP_FLAGS once a split has written its flags to ws."""
    if not isinstance(t, GroupedPlanes):
        ld = _pitch(t, where)
        if len(t.shape) == 2 and _dtype(t, where) == BF16 and src is None and _tma_ok(t, ld):
            return t, t.data_ptr(), ld, 0, 1, keep
        t, keep = _split(t, ends, src, None, ws, stream, keep), KEEP_FLAGS
    elif src is not None or not t.padded:
        _bad(where, "a plane set of token rows, already gathered, is needed")
    else:
        _whole_planes(t, ends.numel(), where)
    return t, t.planes.data_ptr(), t.ld, 1, t.nslices, keep


def grouped_wgrad(A, B, ends, srcA=None, srcB=None, D=None, ws=None, stream=None):
    """D_g = A[srcA]^T B[srcB] over the rows of group g: D [G, M, N].  The
    gradient of W is grouped_wgrad(X, dY) for OP_N and grouped_wgrad(dY, X)
    for OP_T.  A and B: token rows of one type, or plane sets of
    grouped_split.  D as Y in grouped_gemm.  Returns (D, ws)."""
    torch, where = _torch(), "grouped_wgrad"
    G, dev = ends.numel(), A.device
    if ws is None:
        ws = _empty(emu_split_workspace_bytes(32), torch.uint8, dev, stream)
    A, pa, lda, apad, Sa, keep = _token_operand(A, ends, srcA, ws, stream, 0, "grouped_wgrad: A")
    B, pb, ldb, bpad, Sb, keep = _token_operand(B, ends, srcB, ws, stream, keep, "grouped_wgrad: B")
    if A.shape[0] != B.shape[0] or Sa != Sb or B.device != dev:
        _bad(where, "A and B have to be token rows, as many and of one type, on one device")
    (rows, M), N, S = A.shape, B.shape[1], Sa
    if D is None:
        D = _empty((G, M, N), torch.float32 if S == 3 else torch.bfloat16, dev, stream)
    dt, ldd = _dtype(D, "grouped_wgrad: D"), _pitch(D, "grouped_wgrad: D", dev)
    if D.shape != (G, M, N) or (S == 3 and dt != F32):
        _bad(where, "D has another shape or type")
    r = _lib.emu_grouped_prodsum_wgrad(S | keep, G, rows, M, N, pa, lda, apad, pb, ldb, bpad,
                                       _ints(ends, G, dev, "grouped_wgrad: ends"), D.data_ptr(), dt, ldd,
                                       D.stride(0) if G > 1 else M * ldd, ws.data_ptr(), ws.numel(),
                                       _raw_stream(stream, dev))
    if r:
        _check(r, "emu_grouped_prodsum_wgrad")
    return D, ws


def w4_matvec(X, Wq, scales, zeros=None, ends=None, Y=None, ws=None, stream=None):
    """emu_w4_matvec: Y[r] = W_g X[r] for the rows r of group g (ends None: one
    matrix Wq [N, K/2] for all rows), W = (codes - zeros) * scales.  Wq uint8
    [G, N, K/2], the even k in the low half of a byte; scales FP32 or BF16 and
    zeros uint8 (None: 8) [G, N, K/group].  X and Y: FP32 or BF16.  For a few
    rows per expert.  ws: emu_w4_workspace_bytes bytes that a caller may keep
    (made here where they are needed); the call's flags are in a given one.
    Returns Y."""
    torch, where = _torch(), "w4_matvec"
    dev, u8 = X.device, torch.uint8
    dt, ldx, (rows, K) = _dtype(X, "w4_matvec: X"), _pitch(X, "w4_matvec: X"), X.shape
    shape, sshape = Wq.shape, scales.shape
    G = 1 if ends is None else ends.numel()
    N, ng = shape[-2], sshape[-1]
    if 2 * shape[-1] != K:
        _bad(where, f"X has {K} columns, the weights {2 * shape[-1]}")
    if len(shape) != (2 if ends is None else 3) or (ends is not None and shape[0] != G):
        _bad(where, f"weights {tuple(shape)} for {G} group(s)")
    group = K // ng if ng else 32
    if group * ng != K or sshape[:-1] != shape[:-1] or (zeros is not None and zeros.shape != sshape):
        _bad(where, "scales or zeros have another shape")
    if Wq.dtype is not u8 or Wq.device != dev or not Wq.is_contiguous() or scales.device != dev or \
            not scales.is_contiguous() or \
            (zeros is not None and (zeros.dtype is not u8 or zeros.device != dev or not zeros.is_contiguous())):
        _bad(where, f"Wq and zeros have to be uint8, all weights contiguous on {dev}")
    if Y is None:
        Y = _empty((rows, N), X.dtype, dev, stream)
    elif Y.shape != (rows, N) or Y.dtype is not X.dtype:
        _bad(where, "Y has another shape or type")
    x = X.data_ptr()
    if ws is None and (dt == F32 or x % 16 or ldx % 8):
        ws = _empty(_lib.emu_w4_workspace_bytes(dt, rows, K), u8, dev, stream)
    r = _lib.emu_w4_matvec(dt, G, rows, N, K, group, x, ldx, Wq.data_ptr(), scales.data_ptr(),
                           _dtype(scales, "w4_matvec: scales"), zeros.data_ptr() if zeros is not None else None,
                           _ints(ends, G, dev, "w4_matvec: ends") if ends is not None else None, Y.data_ptr(),
                           _pitch(Y, "w4_matvec: Y", dev), ws.data_ptr() if ws is not None else None,
                           ws.numel() if ws is not None else 0, _raw_stream(stream, dev))
    if r:
        _check(r, "emu_w4_matvec")
    return Y


Route = collections.namedtuple("Route", "weights experts slots rows ends")


def route(logits, k: int, renorm: bool = True, ws=None, stream=None):
    """emu_route: the k experts of each token (ties: the lower index), their
    softmax weights over the chosen (renorm) or all experts, and the order of
    the assignments by expert.  Returns (Route(weights, experts, slots [T, k],
    rows [T k], ends [E]), ws): rows and ends are src and ends of grouped_gemm,
    slots and weights those of rows_combine."""
    torch = _torch()
    dt, ldl = _dtype(logits, "route"), _pitch(logits, "route")
    (T, E), dev, i32 = logits.shape, logits.device, torch.int32
    if ws is None:
        ws = _empty(emu_route_workspace_bytes(T, E, k), torch.uint8, dev, stream)
    out = Route(_empty((T, k), torch.float32, dev, stream), _empty((T, k), i32, dev, stream),
                _empty((T, k), i32, dev, stream), _empty(T * k, i32, dev, stream), _empty(E, i32, dev, stream))
    r = _lib.emu_route(dt, T, E, k, int(renorm), logits.data_ptr(), ldl, out[0].data_ptr(), out[1].data_ptr(),
                         out[2].data_ptr(), out[3].data_ptr(), out[4].data_ptr(), ws.data_ptr(), ws.numel(),
                         _raw_stream(stream, dev))
    if r:
        _check(r, "emu_route")
    return out, ws


def _float_pairs(t, shape, device, where):
    """Address of a contiguous float32 tensor of this shape (None: none)."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not _torch().float32 or t.device != device or not t.is_contiguous():
        _bad(where, f"a contiguous float32 tensor {tuple(shape)} on {device} is needed")
    return t.data_ptr()


def route_backward(logits, experts, dweights, renorm: bool = True, dlogits=None, stream=None):
    """emu_route_backward: the logits' gradients from those of route's weights."""
    where = "route_backward"
    dt, (T, E), k, dev = _dtype(logits, where), logits.shape, experts.shape[1], logits.device
    if dlogits is None:
        dlogits = _empty((T, E), logits.dtype, dev, stream)
    elif dlogits.shape != logits.shape or dlogits.dtype is not logits.dtype:
        _bad(where, "dlogits differ from logits")
    r = _lib.emu_route_backward(dt, T, E, k, int(renorm), logits.data_ptr(), _pitch(logits, where),
                                  _ints(experts, T * k, dev, "route_backward: experts"),
                                  _float_pairs(dweights, experts.shape, dev, "route_backward: dweights"),
                                  dlogits.data_ptr(), _pitch(dlogits, where, dev), _raw_stream(stream, dev))
    if r:
        _check(r, "emu_route_backward")
    return dlogits


def rows_combine(Y, slots, weights=None, O=None, stream=None):
    """emu_rows_combine: O[t] = sum_j weights[t, j] Y[slots[t, j]] (weights None: 1)."""
    where = "rows_combine"
    dt, ldy, shape, (yrows, cols), dev = _dtype(Y, where), _pitch(Y, where), slots.shape, Y.shape, Y.device
    T, k = shape
    if O is None:
        O = _empty((T, cols), Y.dtype, dev, stream)
    elif O.shape != (T, cols) or O.dtype is not Y.dtype:
        _bad(where, "O has another shape or type")
    r = _lib.emu_rows_combine(dt, T, k, cols, Y.data_ptr(), yrows, ldy, _ints(slots, T * k, dev, "rows_combine: slots"),
                                _float_pairs(weights, shape, dev, "rows_combine: weights"), O.data_ptr(),
                                _pitch(O, "rows_combine: O", dev), _raw_stream(stream, dev))
    if r:
        _check(r, "emu_rows_combine")
    return O


def rows_combine_backward(dO, Y, slots, weights=None, dY=None, stream=None):
    """emu_rows_combine_backward: (dY, dweights) of rows_combine(Y, slots,
    weights); dweights is None without weights.  No two slots may name the
    same row.  Rows that no slot names are zero in a dY made here, and left as
    they are in a given one."""
    where = "rows_combine_backward"
    dt, shape, (yrows, cols), dev = _dtype(Y, where), slots.shape, Y.shape, Y.device
    T, k = shape
    if dO.shape != (T, cols) or dO.dtype is not Y.dtype:
        _bad(where, "dO has another shape or type")
    full = dY is None
    if full:
        dY = _empty((yrows, cols), Y.dtype, dev, stream)
        ws = _empty(yrows, _torch_module.int32, dev, stream)
    elif dY.shape != Y.shape or dY.dtype is not Y.dtype:
        _bad(where, "dY differs from Y")
    dw = _empty((T, k), _torch_module.float32, dev, stream) if weights is not None else None
    args = (dt, T, k, cols, dO.data_ptr(), _pitch(dO, "rows_combine_backward: dO", dev), Y.data_ptr(), yrows,
            _pitch(Y, where), _ints(slots, T * k, dev, "rows_combine_backward: slots"),
            _float_pairs(weights, shape, dev, "rows_combine_backward: weights"), dY.data_ptr(),
            _pitch(dY, "rows_combine_backward: dY", dev), dw.data_ptr() if dw is not None else None)
    if full:
        r = _lib.emu_rows_combine_backward_full(*args, ws.data_ptr(), 4 * yrows, _raw_stream(stream, dev))
    else:
        r = _lib.emu_rows_combine_backward(*args, _raw_stream(stream, dev))
    if r:
        _check(r, "emu_rows_combine_backward")
    return dY, dw
