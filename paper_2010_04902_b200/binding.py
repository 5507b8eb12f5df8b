"""Thin ctypes binding over libbz.so: one Python function per C entry point, same names minus the
``bz_`` prefix.  It only marshals arguments (pointers, sizes, the current CUDA stream) - every step
of the aggregation runs in the library's kernels.  There is no fallback: a missing library or a
non-zero status raises.

Device arrays are torch CUDA tensors (torch is used for allocation and streams only).
"""
from __future__ import annotations

import ctypes
import math
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libbz.so")

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_PRECONDITION, ERR_WORKSPACE, ERR_BUDGET, ERR_CUDA = -1, -2, -3, -4, -5, -6
OP_PAIRDIST, OP_MULTIKRUM, OP_BULYAN, OP_WORST_CASE, OP_VOTE_MEDIAN_HOST, OP_WORST_CASE_MOLS, OP_VOTE_VECTORWISE = 1, 2, 3, 4, 5, 6, 7
MAX_R, MAX_F = 15, 128
STATUS_RECOMPUTED, STATUS_STOPPED_EARLY = 1, 2
F32, F16, BF16 = 0, 1, 2
ACT_SILU, ACT_GELU_TANH, ACT_GELU, ACT_RELU = range(4)
MAX_DISTANCE, MAX_TOP = 2048, 1024
NORM_RMS, NORM_LAYER = 0, 1
MAX_WIDTH = 16384
GLU_FEW = 32                # up to so many rows bz_glu needs no workspace
PATH_NONE, PATH_STAGED, PATH_REGISTERS, PATH_GENERIC, PATH_TENSOR, PATH_FP32, PATH_FP32_FUSED, PATH_FP64 = range(8)


class BzError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        msg = "%s failed: %s (%d)" % (what, status_string(status), status)
        if status == ERR_CUDA:
            msg += " - " + last_cuda_error()
        super().__init__(msg)


_lib = None

_c_int, _c_i64, _c_sz, _c_vp, _c_u64 = ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_uint64
_c_f, _c_d = ctypes.c_float, ctypes.c_double

_SIGNATURES = {
    "bz_assign_mols": (_c_int, [_c_int, _c_int, _c_vp, _c_vp, _c_vp]),
    "bz_assign_ramanujan": (_c_int, [_c_int, _c_int, _c_vp, _c_vp, _c_vp]),
    "bz_vote": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_i64, _c_i64, _c_vp, _c_i64, _c_vp]),
    "bz_vote_median_rows": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_vp, _c_vp]),
    "bz_vote_rows": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_vp, _c_i64, _c_vp]),
    "bz_vote_vectorwise": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_i64, _c_i64, _c_vp, _c_i64, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_vote_clusters": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_i64, _c_i64, ctypes.c_float, ctypes.c_float, _c_vp, _c_i64, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_median": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_vp, _c_vp]),
    "bz_vote_median": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_i64, _c_i64, _c_vp, _c_vp]),
    "bz_vote_median_host": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_vote_median_update": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_i64, _c_i64, _c_vp, _c_vp, ctypes.c_float,
                                       ctypes.c_float, _c_vp, _c_vp]),
    "bz_model_update": (_c_int, [_c_vp, _c_i64, _c_vp, _c_vp, ctypes.c_float, ctypes.c_float, _c_vp]),
    "bz_pairdist": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_pairdist_static": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_vp, _c_vp]),
    "bz_krum_select": (_c_int, [_c_vp, _c_int, _c_int, _c_int, _c_vp, _c_vp]),
    "bz_mean_rows": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_vp, _c_int, _c_vp, _c_vp]),
    "bz_multikrum": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_int, _c_int, _c_vp, _c_vp, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_bulyan_select": (_c_int, [_c_vp, _c_int, _c_int, _c_vp, _c_vp]),
    "bz_trimmed_mean": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_vp, _c_int, _c_int, _c_vp, _c_vp]),
    "bz_bulyan": (_c_int, [_c_vp, _c_int, _c_i64, _c_i64, _c_int, _c_vp, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_worst_case": (_c_int, [_c_vp, _c_int, _c_int, _c_int, _c_int, _c_u64, _c_vp, _c_vp, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_worst_case_part": (_c_int, [_c_vp, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_u64, _c_vp, _c_vp, _c_vp, _c_vp, _c_sz,
                                    _c_vp]),
    "bz_vote_pairdist": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_i64, _c_i64, _c_vp, _c_i64, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_vote_multikrum": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_i64, _c_i64, _c_int, _c_int, _c_vp, _c_i64, _c_vp, _c_vp,
                                   _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_vote_bulyan": (_c_int, [_c_vp, _c_int, _c_int, _c_i64, _c_i64, _c_i64, _c_int, _c_vp, _c_i64, _c_vp, _c_vp, _c_vp,
                                _c_sz, _c_vp]),
    "bz_worst_case_mols": (_c_int, [_c_int, _c_int, _c_int, _c_u64, _c_vp, _c_vp, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_worst_case_mols_part": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_u64, _c_vp, _c_vp, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_mols_orbit_count": (_c_int, [_c_int, _c_int, _c_int, _c_vp]),
    "bz_workspace_bytes": (_c_sz, [_c_int, _c_int, _c_int, _c_i64, _c_int, _c_int]),
    "bz_status_string": (ctypes.c_char_p, [_c_int]),
    "bz_last_cuda_error": (ctypes.c_char_p, []),
    "bz_kernel_launch_count": (_c_u64, []),
    "bz_pipeline_timeouts": (_c_int, [_c_vp]),
    "bz_pairdist_status": (_c_int, [_c_vp, _c_int, _c_vp, _c_vp]),
    "bz_debug_stall_pipeline": (_c_int, [_c_int]),
    "bz_last_path": (_c_int, []),
    "bz_stream_probe": (_c_int, [_c_vp, _c_sz, _c_int, _c_vp, _c_vp]),
    "bz_glu": (_c_int, [_c_vp, _c_i64, _c_vp, _c_vp, _c_i64, _c_i64, _c_i64, _c_i64, _c_int, _c_int, _c_vp, _c_i64, _c_vp, _c_vp, _c_sz,
                        _c_vp]),
    "bz_glu_backward": (_c_int, [_c_vp, _c_i64, _c_vp, _c_vp, _c_i64, _c_vp, _c_vp, _c_i64, _c_i64, _c_i64, _c_i64, _c_int, _c_int, _c_vp,
                                 _c_i64, _c_vp, _c_vp, _c_i64, _c_int, _c_vp, _c_sz, _c_vp]),
    "bz_glu_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64, _c_int, _c_int]),
    "bz_bias_softmax": (_c_int, [_c_vp, _c_vp, _c_int, _c_i64, _c_i64, _c_i64, _c_i64, _c_vp, _c_int, _c_int, _c_int, _c_int, _c_f, _c_vp,
                                 _c_vp, _c_vp, _c_vp, _c_vp, _c_vp]),
    "bz_bias_softmax_backward": (_c_int, [_c_vp, _c_vp, _c_int, _c_i64, _c_i64, _c_i64, _c_i64, _c_vp, _c_int, _c_int, _c_int, _c_int, _c_f,
                                          _c_vp, _c_vp, _c_vp, _c_vp, _c_vp, _c_vp, _c_vp, _c_vp, _c_vp, _c_sz, _c_vp]),
    "bz_bias_softmax_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64, _c_i64, _c_int]),
    "bz_distill": (_c_int, [_c_vp, _c_i64, _c_int, _c_i64, _c_i64, _c_vp, _c_vp, _c_int, _c_f, _c_vp, _c_vp, _c_vp, _c_vp, _c_i64, _c_vp]),
    "bz_distill_backward": (_c_int, [_c_vp, _c_i64, _c_int, _c_i64, _c_i64, _c_vp, _c_vp, _c_int, _c_f, _c_vp, _c_vp, _c_vp, _c_i64, _c_vp]),
    "bz_policy": (_c_int, [_c_vp, _c_i64, _c_int, _c_i64, _c_i64, _c_vp, _c_vp, _c_vp, _c_vp, _c_f, _c_f, _c_f, _c_f, _c_vp, _c_vp, _c_vp, _c_vp,
                           _c_vp, _c_i64, _c_vp]),
    "bz_preference": (_c_int, [_c_vp, _c_i64, _c_int, _c_i64, _c_i64, _c_vp, _c_vp, _c_vp, _c_i64, _c_f, _c_f, _c_f, _c_f, _c_int, _c_vp, _c_vp,
                               _c_vp, _c_vp, _c_vp, _c_vp, _c_i64, _c_vp]),
    "bz_token_loss_backward": (_c_int, [_c_vp, _c_i64, _c_int, _c_i64, _c_i64, _c_vp, _c_f, _c_vp, _c_vp, _c_i64, _c_vp, _c_i64, _c_vp]),
    "bz_dropout": (_c_int, [_c_vp, _c_i64, _c_int, _c_i64, _c_i64, _c_d, _c_vp, _c_vp, _c_i64, _c_vp]),
    "bz_join": (_c_int, [_c_vp, _c_i64, _c_vp, _c_i64, _c_int, _c_i64, _c_i64, _c_int, _c_f, _c_vp, _c_vp, _c_i64, _c_f, _c_f, _c_d, _c_vp, _c_vp,
                         _c_vp, _c_i64, _c_vp, _c_i64, _c_vp, _c_vp]),
    "bz_join_backward": (_c_int, [_c_vp, _c_i64, _c_vp, _c_i64, _c_int, _c_i64, _c_i64, _c_int, _c_vp, _c_vp, _c_i64, _c_f, _c_f, _c_d, _c_vp,
                                  _c_vp, _c_vp, _c_vp, _c_i64, _c_vp, _c_i64, _c_vp, _c_i64, _c_vp, _c_i64, _c_vp, _c_vp, _c_vp, _c_vp, _c_sz,
                                  _c_vp]),
    "bz_join_workspace_bytes": (_c_sz, [_c_i64, _c_i64, _c_i64]),
}

EXPORTS = sorted(_SIGNATURES)


def lib() -> ctypes.CDLL:
    """Load libbz.so (built in-tree by ``python -m paper_2010_04902_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libbz.so is missing at %s: run `python -m paper_2010_04902_b200.build` "
                              "(there is no CPU fallback)" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().bz_status_string(status).decode()


def last_cuda_error() -> str:
    return lib().bz_last_cuda_error().decode()


def kernel_launch_count() -> int:
    return int(lib().bz_kernel_launch_count())


def pipeline_timeouts() -> int:
    """Barrier waits that ran out inside the TMA-staged kernels since the library was loaded (0 when healthy)."""
    n = ctypes.c_uint(0)
    _check(lib().bz_pipeline_timeouts(ctypes.addressof(n)), "bz_pipeline_timeouts")
    return int(n.value)


def stream_probe(buf: torch.Tensor, checksum: torch.Tensor | None = None, staged: bool = False) -> torch.Tensor:
    """bz_stream_probe: XOR of the 64-bit words of `buf` (any dtype, contiguous), read once from device memory
    (staged: through the bulk-copy engine and shared memory instead of plain loads)."""
    if not buf.is_cuda or not buf.is_contiguous():
        raise TypeError("buf must be a contiguous CUDA tensor")
    if checksum is None:
        checksum = torch.zeros(1, dtype=torch.int64, device=buf.device)
    _check(lib().bz_stream_probe(buf.data_ptr(), buf.numel() * buf.element_size(), 1 if staged else 0,
                                 _dev(checksum, torch.int64, "checksum"), _stream()), "bz_stream_probe")
    return checksum


def last_path() -> int:
    """PATH_* of the kernel family this thread's last call dispatched to."""
    return int(lib().bz_last_path())


def pairdist_status(workspace: torch.Tensor, f: int) -> int:
    """STATUS_* bits of the distance stage of the last call that used `workspace` (synchronises the stream)."""
    st = ctypes.c_int32(0)
    _check(lib().bz_pairdist_status(_dev(workspace, torch.uint8, "workspace"), f, ctypes.addressof(st), _stream()),
           "bz_pairdist_status")
    return int(st.value)


def debug_stall_pipeline(on: int) -> None:
    """Testing aid: make the bounded waits of the tensor-core kernels (distances, gated block) run out (see bz.h)."""
    _check(lib().bz_debug_stall_pipeline(int(on)), "bz_debug_stall_pipeline")


def _check(status: int, what: str):
    if status != OK:
        raise BzError(status, what)


def _stream() -> int:
    # torch.cuda.current_stream().cuda_stream without building the stream object (3.2 -> 0.3 us a call)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError("%s must be a CUDA tensor of dtype %s" % (name, dtype))
    return t.data_ptr()


def _room(workspace: torch.Tensor):
    """(address, bytes) of a workspace: contiguous device memory of any type."""
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous CUDA tensor")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _rows(t: torch.Tensor, name: str):
    """(f, d, ld) of a [f][d] tensor whose last dimension is contiguous."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("%s must be [f][d] with unit stride along d" % name)
    f, d = t.shape
    return f, d, (max(d, t.stride(0)) if f > 1 else d)


def _replicas(t: torch.Tensor):
    """(r, f, d, ld_file, ld_replica) of a [r][f][d] tensor whose last dimension is contiguous."""
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError("replicas must be [r][f][d] with unit stride along d")
    r, f, d = t.shape
    ld_file = max(d, t.stride(1)) if f > 1 else d
    ld_rep = max(d, t.stride(0)) if r > 1 else f * ld_file
    return r, f, d, ld_file, ld_rep


def workspace_bytes(op: int, r: int = 0, f: int = 0, d: int = 0, c: int = 0, m: int = 0) -> int:
    return int(lib().bz_workspace_bytes(op, r, f, d, c, m))


def alloc_workspace(op: int, r: int = 0, f: int = 0, d: int = 0, c: int = 0, m: int = 0, device="cuda") -> torch.Tensor:
    n = workspace_bytes(op, r, f, d, c, m)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


# --------------------------------------------------------------------------------------------- host

def assign_mols(l: int, r: int):
    """Algorithm 2.  Returns numpy (worker_files[K][l], file_workers[f][r], worker_mask[K] or None)."""
    K, f = max(r * l, 1), max(l * l, 1)
    wf = np.zeros((K, max(l, 1)), np.int32)
    fw = np.zeros((f, max(r, 1)), np.int32)
    mask = np.zeros(K, np.uint64) if l * l <= 64 else None
    st = lib().bz_assign_mols(l, r, wf.ctypes.data, fw.ctypes.data, mask.ctypes.data if mask is not None else None)
    _check(st, "bz_assign_mols(l=%d, r=%d)" % (l, r))
    return wf, fw, mask


def ramanujan_dims(m: int, s: int):
    """(K, f, l, r) of Eq. (7) for the Ramanujan construction with parameters (m, s)."""
    return (m * s, s * s, s, m) if m < s else (s * s, m * s, m, s)


def assign_ramanujan(m: int, s: int):
    """Sec. 4.2.1.  Returns numpy (worker_files[K][l], file_workers[f][r], worker_mask[K] or None)."""
    K, f, l, r = ramanujan_dims(max(m, 1), max(s, 1))
    wf = np.zeros((K, l), np.int32)
    fw = np.zeros((f, r), np.int32)
    mask = np.zeros(K, np.uint64) if f <= 64 else None
    st = lib().bz_assign_ramanujan(m, s, wf.ctypes.data, fw.ctypes.data, mask.ctypes.data if mask is not None else None)
    _check(st, "bz_assign_ramanujan(m=%d, s=%d)" % (m, s))
    return wf, fw, mask


def worst_case(worker_mask, f: int, r: int, q: int, max_subsets: int = 0, workspace: torch.Tensor | None = None):
    """Exhaustive c_max^(q).  Returns (c_max, argmax[q] numpy, n_subsets)."""
    mask = np.ascontiguousarray(worker_mask, np.uint64)
    K = int(mask.shape[0])
    ws = workspace if workspace is not None else alloc_workspace(OP_WORST_CASE, r, f)
    cmax = ctypes.c_int32(0)
    n = ctypes.c_uint64(0)
    arg = np.zeros(max(q, 1), np.int32)
    st = lib().bz_worst_case(mask.ctypes.data, K, f, r, q, max_subsets, ctypes.addressof(cmax), arg.ctypes.data,
                             ctypes.addressof(n), *_room(ws), _stream())
    _check(st, "bz_worst_case(K=%d, q=%d)" % (K, q))
    return int(cmax.value), arg[:q].copy(), int(n.value)


def worst_case_part(worker_mask, f: int, r: int, q: int, part: int, parts: int, max_subsets: int = 0,
                    workspace: torch.Tensor | None = None):
    """bz_worst_case_part: share `part` of `parts` of the exhaustive search.  Returns (c_max, argmax[q] numpy,
    n_subsets); c_max is -1 for a share that received nothing."""
    mask = np.ascontiguousarray(worker_mask, np.uint64)
    K = int(mask.shape[0])
    ws = workspace if workspace is not None else alloc_workspace(OP_WORST_CASE, r, f)
    cmax = ctypes.c_int32(0)
    n = ctypes.c_uint64(0)
    arg = np.zeros(max(q, 1), np.int32)
    st = lib().bz_worst_case_part(mask.ctypes.data, K, f, r, q, part, parts, max_subsets, ctypes.addressof(cmax),
                                  arg.ctypes.data, ctypes.addressof(n), *_room(ws), _stream())
    _check(st, "bz_worst_case_part(K=%d, q=%d, part %d of %d)" % (K, q, part, parts))
    return int(cmax.value), arg[:q].copy(), int(n.value)


def worst_case_mols(l: int, r: int, q: int, max_subsets: int = 0, workspace: torch.Tensor | None = None):
    """bz_worst_case_mols: c_max^(q) of the placement assign_mols(l, r), one set per translation orbit.
    Returns (c_max, argmax[q] numpy, n_orbits)."""
    ws = workspace if workspace is not None else alloc_workspace(OP_WORST_CASE_MOLS, r, l * l)
    cmax = ctypes.c_int32(0)
    n = ctypes.c_uint64(0)
    arg = np.zeros(max(q, 1), np.int32)
    st = lib().bz_worst_case_mols(l, r, q, max_subsets, ctypes.addressof(cmax), arg.ctypes.data, ctypes.addressof(n),
                                  *_room(ws), _stream())
    _check(st, "bz_worst_case_mols(l=%d, r=%d, q=%d)" % (l, r, q))
    return int(cmax.value), arg[:q].copy(), int(n.value)


def worst_case_mols_part(l: int, r: int, q: int, part: int, parts: int, max_subsets: int = 0,
                         workspace: torch.Tensor | None = None):
    """bz_worst_case_mols_part: share `part` of `parts` of the orbit search.  Returns (c_max, argmax[q] numpy, n_orbits);
    c_max is -1 for a share that received nothing."""
    ws = workspace if workspace is not None else alloc_workspace(OP_WORST_CASE_MOLS, r, l * l)
    cmax = ctypes.c_int32(0)
    n = ctypes.c_uint64(0)
    arg = np.zeros(max(q, 1), np.int32)
    st = lib().bz_worst_case_mols_part(l, r, q, part, parts, max_subsets, ctypes.addressof(cmax), arg.ctypes.data,
                                       ctypes.addressof(n), *_room(ws), _stream())
    _check(st, "bz_worst_case_mols_part(l=%d, r=%d, q=%d, part %d of %d)" % (l, r, q, part, parts))
    return int(cmax.value), arg[:q].copy(), int(n.value)


def mols_orbit_count(l: int, r: int, q: int) -> int:
    n = ctypes.c_uint64(0)
    _check(lib().bz_mols_orbit_count(l, r, q, ctypes.addressof(n)), "bz_mols_orbit_count")
    return int(n.value)


# --------------------------------------------------------------------------------------------- device

def vote(replicas: torch.Tensor, voted: torch.Tensor | None = None) -> torch.Tensor:
    r, f, d, ld_file, ld_rep = _replicas(replicas)
    if voted is None:
        voted = torch.empty((f, d), dtype=torch.float32, device=replicas.device)
    vf, vd, ld_v = _rows(voted, "voted")
    if (vf, vd) != (f, d):
        raise ValueError("voted must be [%d][%d]" % (f, d))
    st = lib().bz_vote(_dev(replicas, torch.float32, "replicas"), r, f, d, ld_file, ld_rep,
                       _dev(voted, torch.float32, "voted"), ld_v, _stream())
    _check(st, "bz_vote")
    return voted


def row_table(worker_buffers, file_workers, worker_files) -> torch.Tensor:
    """Device table of r*f row pointers for bz_vote_median_rows / bz_vote_rows from what the workers sent:
    worker_buffers[u] is a CUDA float32 tensor [l][d] holding worker u's gradients in the order of
    worker_files[u]; entry k*f + i of the table points at the gradient worker file_workers[i][k] returned
    for file i.  The buffers must stay alive while the table is in use."""
    f, r = len(file_workers), len(file_workers[0])
    ptrs = []
    for k in range(r):
        for i in range(f):
            u = int(file_workers[i][k])
            slot = [int(x) for x in worker_files[u]].index(i)
            row = worker_buffers[u][slot]
            if row.dtype != torch.float32 or not row.is_cuda or row.stride(0) != 1:
                raise ValueError("worker buffers must be CUDA float32 tensors with contiguous rows")
            ptrs.append(row.data_ptr())
    return torch.tensor(ptrs, dtype=torch.int64, device=worker_buffers[0].device)


def vote_median_rows(table: torch.Tensor, r: int, f: int, d: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """bz_vote_median_rows on a table made by row_table()."""
    if table.dtype != torch.int64 or not table.is_cuda or table.numel() != r * f:
        raise ValueError("table must be a CUDA int64 tensor of r*f pointers")
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=table.device)
    st = lib().bz_vote_median_rows(table.data_ptr(), r, f, d, _dev(out, torch.float32, "out"), _stream())
    _check(st, "bz_vote_median_rows")
    return out


def vote_rows(table: torch.Tensor, r: int, f: int, d: int, voted: torch.Tensor | None = None) -> torch.Tensor:
    """bz_vote_rows on a table made by row_table()."""
    if table.dtype != torch.int64 or not table.is_cuda or table.numel() != r * f:
        raise ValueError("table must be a CUDA int64 tensor of r*f pointers")
    if voted is None:
        voted = torch.empty((f, d), dtype=torch.float32, device=table.device)
    _, _, ld_v = _rows(voted, "voted")
    st = lib().bz_vote_rows(table.data_ptr(), r, f, d, _dev(voted, torch.float32, "voted"), ld_v, _stream())
    _check(st, "bz_vote_rows")
    return voted


def vote_vectorwise(replicas: torch.Tensor, voted: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """bz_vote_vectorwise: the vote of Eq. (3) on whole gradients.  Returns (voted[f][d], winner[f])."""
    r, f, d, ld_file, ld_rep = _replicas(replicas)
    if voted is None:
        voted = torch.empty((f, d), dtype=torch.float32, device=replicas.device)
    vf, vd, ld_v = _rows(voted, "voted")
    if (vf, vd) != (f, d):
        raise ValueError("voted must be [%d][%d]" % (f, d))
    ws = workspace if workspace is not None else alloc_workspace(OP_VOTE_VECTORWISE, r, f, d, device=replicas.device)
    winner = torch.empty(f, dtype=torch.int32, device=replicas.device)
    st = lib().bz_vote_vectorwise(_dev(replicas, torch.float32, "replicas"), r, f, d, ld_file, ld_rep,
                                  _dev(voted, torch.float32, "voted"), ld_v, winner.data_ptr(), *_room(ws),
                                  _stream())
    _check(st, "bz_vote_vectorwise")
    return voted, winner


def vote_clusters(replicas: torch.Tensor, abs_tol: float, rel_tol: float, voted: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None):
    """bz_vote_clusters: the whole-vector vote with agreement up to a tolerance.  Returns (voted[f][d], winner[f])."""
    r, f, d, ld_file, ld_rep = _replicas(replicas)
    if voted is None:
        voted = torch.empty((f, d), dtype=torch.float32, device=replicas.device)
    vf, vd, ld_v = _rows(voted, "voted")
    if (vf, vd) != (f, d):
        raise ValueError("voted must be [%d][%d]" % (f, d))
    ws = workspace if workspace is not None else alloc_workspace(OP_VOTE_VECTORWISE, r, f, d, device=replicas.device)
    winner = torch.empty(f, dtype=torch.int32, device=replicas.device)
    st = lib().bz_vote_clusters(_dev(replicas, torch.float32, "replicas"), r, f, d, ld_file, ld_rep, float(abs_tol),
                                float(rel_tol), _dev(voted, torch.float32, "voted"), ld_v, winner.data_ptr(), *_room(ws), _stream())
    _check(st, "bz_vote_clusters")
    return voted, winner


def median(voted: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    f, d, ld = _rows(voted, "voted")
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=voted.device)
    st = lib().bz_median(_dev(voted, torch.float32, "voted"), f, d, ld, _dev(out, torch.float32, "out"), _stream())
    _check(st, "bz_median")
    return out


def vote_median(replicas: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    r, f, d, ld_file, ld_rep = _replicas(replicas)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=replicas.device)
    st = lib().bz_vote_median(_dev(replicas, torch.float32, "replicas"), r, f, d, ld_file, ld_rep,
                              _dev(out, torch.float32, "out"), _stream())
    _check(st, "bz_vote_median")
    return out


def _state(t, d: int, name: str):
    if t is None:
        return None
    if t.dim() != 1 or t.numel() != d or not t.is_contiguous():
        raise TypeError("%s must be a contiguous [d] tensor" % name)
    return _dev(t, torch.float32, name)


def vote_median_update(replicas: torch.Tensor, w: torch.Tensor, eta: float, velocity: torch.Tensor | None = None,
                       mu: float = 0.0, out: torch.Tensor | None = None) -> None:
    """bz_vote_median_update: aggregate and apply Eq. (1) to w (and velocity) in place; `out`, when given,
    also receives the aggregate."""
    r, f, d, ld_file, ld_rep = _replicas(replicas)
    st = lib().bz_vote_median_update(_dev(replicas, torch.float32, "replicas"), r, f, d, ld_file, ld_rep,
                                     _state(w, d, "w"), _state(velocity, d, "velocity"), eta, mu,
                                     _state(out, d, "out"), _stream())
    _check(st, "bz_vote_median_update")


def model_update(g: torch.Tensor, w: torch.Tensor, eta: float, velocity: torch.Tensor | None = None,
                 mu: float = 0.0) -> None:
    d = g.numel()
    st = lib().bz_model_update(_state(g, d, "g"), d, _state(w, d, "w"), _state(velocity, d, "velocity"), eta, mu,
                               _stream())
    _check(st, "bz_model_update")


def vote_median_host(replicas_host: torch.Tensor, out_host: torch.Tensor, workspace: torch.Tensor) -> torch.Tensor:
    """replicas_host: contiguous CPU [r][f][d] (pin it for full copy speed); out_host: CPU [d]."""
    if replicas_host.is_cuda or out_host.is_cuda or not replicas_host.is_contiguous() or not out_host.is_contiguous():
        raise TypeError("replicas_host / out_host must be contiguous CPU tensors")
    if replicas_host.dtype != torch.float32 or out_host.dtype != torch.float32:
        raise TypeError("float32 expected")
    r, f, d = replicas_host.shape
    st = lib().bz_vote_median_host(replicas_host.data_ptr(), r, f, d, out_host.data_ptr(), *_room(workspace), _stream())
    _check(st, "bz_vote_median_host")
    return out_host


def pairdist(voted: torch.Tensor, workspace: torch.Tensor | None = None, dist: torch.Tensor | None = None) -> torch.Tensor:
    f, d, ld = _rows(voted, "voted")
    ws = workspace if workspace is not None else alloc_workspace(OP_PAIRDIST, 0, f, d, device=voted.device)
    if dist is None:
        dist = torch.empty((f, f), dtype=torch.float64, device=voted.device)
    st = lib().bz_pairdist(_dev(voted, torch.float32, "voted"), f, d, ld, _dev(dist, torch.float64, "dist"),
                           *_room(ws), _stream())
    _check(st, "bz_pairdist")
    return dist


STATIC_SCRATCH_BYTES = 4 << 20
ERR_STATIC_LIMIT = -7


def pairdist_static(voted: torch.Tensor, dist: torch.Tensor) -> torch.Tensor:
    """bz_pairdist_static: the distance matrix for a caller that cannot supply (or allocate) a device
    workspace - for example code running under a frozen memory plan or a fixed memory budget.  The
    scratch is a 4 MiB array inside the library; `dist` ([f][f] float64) must already exist.  Shapes
    that need more scratch (f > 84) raise with status ERR_STATIC_LIMIT.  Calls share that
    array: do not let two of them run on the GPU at the same time."""
    f, d, ld = _rows(voted, "voted")
    st = lib().bz_pairdist_static(_dev(voted, torch.float32, "voted"), f, d, ld, _dev(dist, torch.float64, "dist"),
                                  _stream())
    _check(st, "bz_pairdist_static")
    return dist


def krum_select(dist: torch.Tensor, c: int, m: int) -> torch.Tensor:
    f = dist.shape[0]
    sel = torch.empty(max(m, 1), dtype=torch.int32, device=dist.device)
    st = lib().bz_krum_select(_dev(dist, torch.float64, "dist"), f, c, m, sel.data_ptr(), _stream())
    _check(st, "bz_krum_select")
    return sel[:m]


def mean_rows(voted: torch.Tensor, selected: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    f, d, ld = _rows(voted, "voted")
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=voted.device)
    st = lib().bz_mean_rows(_dev(voted, torch.float32, "voted"), f, d, ld, _dev(selected, torch.int32, "selected"),
                            selected.numel(), _dev(out, torch.float32, "out"), _stream())
    _check(st, "bz_mean_rows")
    return out


def multikrum(voted: torch.Tensor, c: int, m: int, workspace: torch.Tensor | None = None,
              out: torch.Tensor | None = None, want_dist: bool = False):
    """Returns (out[d], selected[m]) or (out, selected, dist) with want_dist."""
    f, d, ld = _rows(voted, "voted")
    ws = workspace if workspace is not None else alloc_workspace(OP_MULTIKRUM, 0, f, d, c, m, device=voted.device)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=voted.device)
    sel = torch.empty(max(m, 1), dtype=torch.int32, device=voted.device)
    dist = torch.empty((f, f), dtype=torch.float64, device=voted.device) if want_dist else None
    st = lib().bz_multikrum(_dev(voted, torch.float32, "voted"), f, d, ld, c, m, _dev(out, torch.float32, "out"),
                            sel.data_ptr(), dist.data_ptr() if dist is not None else None, *_room(ws),
                            _stream())
    _check(st, "bz_multikrum")
    return (out, sel[:m], dist) if want_dist else (out, sel[:m])


def bulyan_select(dist: torch.Tensor, c: int) -> torch.Tensor:
    f = dist.shape[0]
    theta = f - 2 * c
    sel = torch.empty(max(theta, 1), dtype=torch.int32, device=dist.device)
    st = lib().bz_bulyan_select(_dev(dist, torch.float64, "dist"), f, c, sel.data_ptr(), _stream())
    _check(st, "bz_bulyan_select")
    return sel[:theta]


def trimmed_mean(voted: torch.Tensor, selected: torch.Tensor, beta: int, out: torch.Tensor | None = None) -> torch.Tensor:
    f, d, ld = _rows(voted, "voted")
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=voted.device)
    st = lib().bz_trimmed_mean(_dev(voted, torch.float32, "voted"), f, d, ld, _dev(selected, torch.int32, "selected"),
                               selected.numel(), beta, _dev(out, torch.float32, "out"), _stream())
    _check(st, "bz_trimmed_mean")
    return out


def bulyan(voted: torch.Tensor, c: int, workspace: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """Returns (out[d], selected[f - 2c])."""
    f, d, ld = _rows(voted, "voted")
    ws = workspace if workspace is not None else alloc_workspace(OP_BULYAN, 0, f, d, c, device=voted.device)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=voted.device)
    theta = f - 2 * c
    sel = torch.empty(max(theta, 1), dtype=torch.int32, device=voted.device)
    st = lib().bz_bulyan(_dev(voted, torch.float32, "voted"), f, d, ld, c, _dev(out, torch.float32, "out"),
                         sel.data_ptr(), *_room(ws), _stream())
    _check(st, "bz_bulyan")
    return out, sel[:max(theta, 0)]


# ------------------------------------------------------------------------- from the replicas in one pass

def _voted_for(replicas: torch.Tensor, voted: torch.Tensor | None):
    r, f, d, ld_file, ld_rep = _replicas(replicas)
    if voted is None:
        voted = torch.empty((f, d), dtype=torch.float32, device=replicas.device)
    vf, vd, ld_v = _rows(voted, "voted")
    if (vf, vd) != (f, d):
        raise ValueError("voted must be [%d][%d]" % (f, d))
    return r, f, d, ld_file, ld_rep, voted, ld_v


def vote_pairdist(replicas: torch.Tensor, voted: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                  dist: torch.Tensor | None = None):
    """bz_vote_pairdist: returns (voted[f][d], dist[f][f])."""
    r, f, d, ld_file, ld_rep, voted, ld_v = _voted_for(replicas, voted)
    ws = workspace if workspace is not None else alloc_workspace(OP_PAIRDIST, 0, f, d, device=replicas.device)
    if dist is None:
        dist = torch.empty((f, f), dtype=torch.float64, device=replicas.device)
    st = lib().bz_vote_pairdist(_dev(replicas, torch.float32, "replicas"), r, f, d, ld_file, ld_rep,
                                _dev(voted, torch.float32, "voted"), ld_v, _dev(dist, torch.float64, "dist"),
                                *_room(ws), _stream())
    _check(st, "bz_vote_pairdist")
    return voted, dist


def vote_multikrum(replicas: torch.Tensor, c: int, m: int, voted: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None, out: torch.Tensor | None = None,
                   dist: torch.Tensor | None = None):
    """bz_vote_multikrum: returns (out[d], selected[m], voted[f][d]); the distance matrix goes to `dist` if given."""
    r, f, d, ld_file, ld_rep, voted, ld_v = _voted_for(replicas, voted)
    ws = workspace if workspace is not None else alloc_workspace(OP_MULTIKRUM, 0, f, d, c, m, device=replicas.device)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=replicas.device)
    sel = torch.empty(max(m, 1), dtype=torch.int32, device=replicas.device)
    st = lib().bz_vote_multikrum(_dev(replicas, torch.float32, "replicas"), r, f, d, ld_file, ld_rep, c, m,
                                 _dev(voted, torch.float32, "voted"), ld_v, _dev(out, torch.float32, "out"),
                                 sel.data_ptr(), None if dist is None else _dev(dist, torch.float64, "dist"),
                                 *_room(ws), _stream())
    _check(st, "bz_vote_multikrum")
    return out, sel[:m], voted


def vote_bulyan(replicas: torch.Tensor, c: int, voted: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """bz_vote_bulyan: returns (out[d], selected[f - 2c], voted[f][d])."""
    r, f, d, ld_file, ld_rep, voted, ld_v = _voted_for(replicas, voted)
    ws = workspace if workspace is not None else alloc_workspace(OP_BULYAN, 0, f, d, c, device=replicas.device)
    if out is None:
        out = torch.empty(d, dtype=torch.float32, device=replicas.device)
    theta = f - 2 * c
    sel = torch.empty(max(theta, 1), dtype=torch.int32, device=replicas.device)
    st = lib().bz_vote_bulyan(_dev(replicas, torch.float32, "replicas"), r, f, d, ld_file, ld_rep, c,
                              _dev(voted, torch.float32, "voted"), ld_v, _dev(out, torch.float32, "out"),
                              sel.data_ptr(), *_room(ws), _stream())
    _check(st, "bz_vote_bulyan")
    return out, sel[:max(theta, 0)], voted


# ------------------------------------------------------------------------------------- a worker's step
#
# These calls record nothing for automatic differentiation: each has its gradient as a call of its own.  The forward calls
# refuse tensors that require a gradient while gradients are recorded, whose gradient would be lost without a word.

_DTYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_Strides = ctypes.c_int64 * 3
_ACTS = {"silu": ACT_SILU, "gelu_tanh": ACT_GELU_TANH, "gelu": ACT_GELU, "relu": ACT_RELU}


def _dtype(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda or t.dtype not in _DTYPES:
        raise TypeError("%s must be a CUDA tensor of float32, float16 or bfloat16" % name)
    return _DTYPES[t.dtype]


def _matrix(t: torch.Tensor, name: str):
    """_rows(), and rows that overlap (an expanded tensor's) are refused: there is no leading dimension for them."""
    if t.dim() != 2:
        raise ValueError("%s must be a matrix" % name)
    (f, d), (ld, one) = t.shape, t.stride()
    if d > 1 and one != 1:
        raise ValueError("%s must have unit stride along its rows" % name)
    if f <= 1:
        return f, d, d
    if ld < d:
        raise ValueError("%s has rows that overlap: make it contiguous" % name)
    return f, d, ld


def _shaped(t: torch.Tensor, shape, dtype, name: str) -> int:
    """Address of a tensor of exactly this shape and type (strides are the caller's business)."""
    if t.shape != shape:
        raise ValueError("%s must be %s" % (name, "".join("[%d]" % n for n in shape)))
    return _dev(t, dtype, name)


def _packed(t, shape, dtype, name: str):
    """Address of a contiguous tensor of this shape and type, or None."""
    if t is None:
        return None
    if t.shape == shape and t.dtype is dtype and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return _shaped(t, shape, dtype, name)


def _like_rows(t: torch.Tensor) -> torch.Tensor:
    """A new tensor of t's shape whose rows are as far apart as t's: the kernels' wide loads and stores need rows that
    sit alike relative to 16-byte boundaries."""
    if t.is_contiguous():
        return torch.empty_like(t)
    n, ld = t.shape[-1], t.stride(-2)
    if t.shape[-2] <= 1 or ld <= n or ld > 2 * n:
        return t.new_empty(t.shape)
    return t.new_empty(t.shape[:-1] + (ld,))[..., :n]


def _unrecorded(what: str, **tensors):
    """Called with the tensors of a forward call of which one at least requires a gradient."""
    if torch.is_grad_enabled():
        raise ValueError("%s: %s requires a gradient, which this call does not record: call it under torch.no_grad() (or inside an "
                         "autograd.Function) and %s_backward for the gradient" % (what, " and ".join(n for n, t in tensors.items() if t.requires_grad), what))


def _act(name: str) -> int:
    try:
        return _ACTS[name]
    except KeyError:
        raise ValueError("act must be one of %s" % ", ".join(sorted(_ACTS))) from None


def _glu_operands(x, w_gate, w_up):
    m, k, ld_x = _matrix(x, "x")
    n, k2, ld_w = _matrix(w_gate, "w_gate")
    if k2 != k or w_up.shape != w_gate.shape:
        raise ValueError("w_gate and w_up must both be [n][%d]" % k)
    if w_up.stride() != w_gate.stride() and _matrix(w_up, "w_up")[2] != ld_w:
        raise ValueError("w_gate and w_up must have the same leading dimension")
    return m, n, k, ld_x, ld_w


def glu_workspace_bytes(m: int, n: int, k: int, dtype=torch.bfloat16, backward: bool = False) -> int:
    return int(lib().bz_glu_workspace_bytes(m, n, k, _DTYPES[dtype], 1 if backward else 0))


def glu(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, act: str = "silu", h: torch.Tensor | None = None,
        preact: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """bz_glu: act(x w_gate^T) * (x w_up^T) for x [m][k], weights [n][k] (float16 or bfloat16).  `preact`, binary32
    [2][m][n], receives both projections for glu_backward."""
    if x.requires_grad or w_gate.requires_grad or w_up.requires_grad:
        _unrecorded("glu", x=x, w_gate=w_gate, w_up=w_up)
    m, n, k, ld_x, ld_w = _glu_operands(x, w_gate, w_up)
    dt = _dtype(x, "x")
    if h is None:
        h, ld_h = x.new_empty((m, n)), n
        ph = h.data_ptr()
    else:
        ph, ld_h = _shaped(h, (m, n), x.dtype, "h"), _matrix(h, "h")[2]
    px, pg, pu = x.data_ptr(), _dev(w_gate, x.dtype, "w_gate"), _dev(w_up, x.dtype, "w_up")
    ws, ws_bytes = None, 0
    if workspace is not None:
        ws, ws_bytes = _room(workspace)
    elif m > GLU_FEW and ((ld_x | ld_w) & 7 or (px | pg | pu) & 15):
        workspace = torch.empty(max(256, lib().bz_glu_workspace_bytes(m, n, k, dt, 0)), dtype=torch.uint8, device=x.device)
        ws, ws_bytes = workspace.data_ptr(), workspace.numel()
    st = lib().bz_glu(px, ld_x, pg, pu, ld_w, m, n, k, dt, _act(act), ph, ld_h, _packed(preact, (2, m, n), torch.float32, "preact"),
                      ws, ws_bytes, _stream())
    if st:
        _check(st, "bz_glu")
    return h


def glu_backward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, preact: torch.Tensor, dh: torch.Tensor,
                 act: str = "silu", dx: torch.Tensor | None = None, dw_gate: torch.Tensor | None = None,
                 dw_up: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """bz_glu_backward: returns (dx, dw_gate, dw_up).  dw_gate and dw_up may be given as float32 tensors (views of a
    gradient row, for instance) to keep the 32-bit sums; new ones have the weights' type."""
    m, n, k, ld_x, ld_w = _glu_operands(x, w_gate, w_up)
    dt = _dtype(x, "x")
    if dx is None:
        dx, ld_dx = x.new_empty((m, k)), k
        p_dx = dx.data_ptr()
    else:
        p_dx, ld_dx = _shaped(dx, (m, k), x.dtype, "dx"), _matrix(dx, "dx")[2]
    if (dw_gate is None) != (dw_up is None):
        raise ValueError("give both dw_gate and dw_up, or neither")
    if dw_gate is None:
        whole = w_gate.is_contiguous()
        dw_gate, dw_up = (torch.empty_like(w_gate), torch.empty_like(w_gate)) if whole else (x.new_empty((n, k)), x.new_empty((n, k)))
        p_dg, p_du, ld_dw, grad = dw_gate.data_ptr(), dw_up.data_ptr(), k, dt
    else:
        p_dg, p_du = _shaped(dw_gate, (n, k), dw_gate.dtype, "dw_gate"), _shaped(dw_up, (n, k), dw_gate.dtype, "dw_up")
        ld_dw, grad = _matrix(dw_gate, "dw_gate")[2], _dtype(dw_gate, "dw_gate")
        if _matrix(dw_up, "dw_up")[2] != ld_dw:
            raise ValueError("dw_gate and dw_up must have the same leading dimension")
    if workspace is None:
        workspace = torch.empty(lib().bz_glu_workspace_bytes(m, n, k, dt, 1), dtype=torch.uint8, device=x.device)
    st = lib().bz_glu_backward(_dev(x, x.dtype, "x"), ld_x, _dev(w_gate, x.dtype, "w_gate"), _dev(w_up, x.dtype, "w_up"), ld_w,
                               _packed(preact, (2, m, n), torch.float32, "preact"), _shaped(dh, (m, n), x.dtype, "dh"),
                               _matrix(dh, "dh")[2], m, n, k, dt, _act(act), p_dx, ld_dx, p_dg, p_du, ld_dw, grad,
                               *_room(workspace), _stream())
    if st:
        _check(st, "bz_glu_backward")
    return dx, dw_gate, dw_up


def _strides(t: torch.Tensor, name: str):
    if t.dim() != 4:
        raise ValueError("%s must be [b][h][tq][tk]" % name)
    a, b, c, one = t.stride()
    if one != 1 and t.shape[3] > 1:
        raise ValueError("%s must have unit stride along tk" % name)
    return _Strides(a, b, c)


def _bias_form(scores, table, max_distance, bidirectional, causal, scale, k_len, q_start):
    """The arguments from scores to q_start of both calls."""
    strides = _strides(scores, "scores")
    b, h, tq, tk = scores.shape
    if table.dim() != 2 or table.shape[1] != h:
        raise ValueError("table must be [buckets][%d]" % h)
    return strides, (scores.data_ptr(), strides, _dtype(scores, "scores"), b, h, tq, tk, _packed(table, table.shape, torch.float32, "table"),
                     table.shape[0], max_distance, 1 if bidirectional else 0, 1 if causal else 0, scale,
                     _packed(k_len, (b,), torch.int32, "k_len"), _packed(q_start, (b,), torch.int32, "q_start"))


def _rows_out(t, like, like_strides, name):
    """(tensor, address, strides) of an output shaped like scores; a new one if t is None."""
    if t is None:
        if like.is_contiguous():
            t = torch.empty_like(like)
            return t, t.data_ptr(), like_strides
        t = _like_rows(like)
        return t, t.data_ptr(), _strides(t, name)
    return t, _shaped(t, like.shape, like.dtype, name), _strides(t, name)


def bias_softmax(scores: torch.Tensor, table: torch.Tensor, max_distance: int = 128, bidirectional: bool = True,
                 causal: bool = False, scale: float = 1.0, k_len: torch.Tensor | None = None,
                 q_start: torch.Tensor | None = None, probs: torch.Tensor | None = None, stats: torch.Tensor | None = None):
    """bz_bias_softmax: softmax over keys of scale * scores [b][h][tq][tk] + table[bucket(key - query)][h].  Returns
    (probs, stats)."""
    if scores.requires_grad or table.requires_grad:
        _unrecorded("bias_softmax", scores=scores, table=table)
    strides, form = _bias_form(scores, table, max_distance, bidirectional, causal, scale, k_len, q_start)
    probs, p_probs, s_probs = _rows_out(probs, scores, strides, "probs")
    if stats is None:
        stats = table.new_empty((*scores.shape[:3], 2))
        p_stats = stats.data_ptr()
    else:
        p_stats = _packed(stats, (*scores.shape[:3], 2), torch.float32, "stats")
    st = lib().bz_bias_softmax(*form, p_probs, s_probs, p_stats, _stream())
    if st:
        _check(st, "bz_bias_softmax")
    if not scores.shape[3]:      # no keys at all: the library has nothing to do, and every row is an empty one
        stats[..., 0], stats[..., 1] = -math.inf, 0.0
    return probs, stats


def bias_softmax_backward(scores: torch.Tensor, table: torch.Tensor, stats: torch.Tensor, dprobs: torch.Tensor,
                          max_distance: int = 128, bidirectional: bool = True, causal: bool = False, scale: float = 1.0,
                          k_len: torch.Tensor | None = None, q_start: torch.Tensor | None = None,
                          dscores: torch.Tensor | None = None, dtable: torch.Tensor | None = None,
                          workspace: torch.Tensor | None = None):
    """bz_bias_softmax_backward: returns (dscores, dtable)."""
    strides, form = _bias_form(scores, table, max_distance, bidirectional, causal, scale, k_len, q_start)
    dscores, p_ds, s_ds = _rows_out(dscores, scores, strides, "dscores")
    if dtable is None:
        dtable = torch.empty_like(table)
    if workspace is None:
        size = lib().bz_bias_softmax_workspace_bytes(*scores.shape, table.shape[0])
        workspace = torch.empty(max(256, size), dtype=torch.uint8, device=scores.device)
    st = lib().bz_bias_softmax_backward(*form, _packed(stats, (*scores.shape[:3], 2), torch.float32, "stats"),
                                        _shaped(dprobs, scores.shape, scores.dtype, "dprobs"), _strides(dprobs, "dprobs"), p_ds, s_ds,
                                        _packed(dtable, table.shape, torch.float32, "dtable"), *_room(workspace),
                                        _stream())
    if st:
        _check(st, "bz_bias_softmax_backward")
    return dscores, dtable


def _teacher(logits, teacher, index):
    m = logits.shape[0]
    if teacher.dim() != 2 or teacher.shape[0] != m:
        raise ValueError("teacher must be [%d][t]" % m)
    return _packed(teacher, teacher.shape, torch.float32, "teacher"), _packed(index, teacher.shape, torch.int32, "index"), teacher.shape[1]


def distill(logits: torch.Tensor, teacher: torch.Tensor, index: torch.Tensor, temperature: float = 1.0,
            dloss: torch.Tensor | None = None, loss: torch.Tensor | None = None, stats: torch.Tensor | None = None,
            dlogits: torch.Tensor | None = None):
    """bz_distill: the loss of each position against the teacher's top logits.  Returns (loss, stats); with `dloss`
    (float32 [m]) or `dlogits` given also the gradient, from the same pass: (loss, stats, dlogits)."""
    if logits.requires_grad:
        _unrecorded("distill", logits=logits)
    m, v, ld = _matrix(logits, "logits")
    dt = _dtype(logits, "logits")
    p_teacher, p_index, top = _teacher(logits, teacher, index)
    grad = dloss is not None or dlogits is not None
    if loss is None:
        loss = teacher.new_empty(m)
    if stats is None:
        stats = teacher.new_empty((m, 2))
    p_d, ld_d = None, 0
    if grad:
        if dlogits is None:
            dlogits = _like_rows(logits)
            p_d, ld_d = dlogits.data_ptr(), dlogits.stride(0) if m > 1 else v
        else:
            p_d, ld_d = _shaped(dlogits, (m, v), logits.dtype, "dlogits"), _matrix(dlogits, "dlogits")[2]
    st = lib().bz_distill(logits.data_ptr(), ld, dt, m, v, p_teacher, p_index, top, temperature,
                          _packed(dloss, (m,), torch.float32, "dloss"), _packed(loss, (m,), torch.float32, "loss"),
                          _packed(stats, (m, 2), torch.float32, "stats"), p_d, ld_d, _stream())
    if st:
        _check(st, "bz_distill")
    return (loss, stats, dlogits) if grad else (loss, stats)


def distill_backward(logits: torch.Tensor, teacher: torch.Tensor, index: torch.Tensor, stats: torch.Tensor,
                     dloss: torch.Tensor | None = None, temperature: float = 1.0,
                     dlogits: torch.Tensor | None = None) -> torch.Tensor:
    """bz_distill_backward: the gradient alone, with stats as distill() returned them."""
    m, v, ld = _matrix(logits, "logits")
    if dlogits is None:
        dlogits = _like_rows(logits)
    st = lib().bz_distill_backward(logits.data_ptr(), ld, _dtype(logits, "logits"), m, v, *_teacher(logits, teacher, index),
                                   temperature, _packed(stats, (m, 2), torch.float32, "stats"),
                                   _packed(dloss, (m,), torch.float32, "dloss"),
                                   _shaped(dlogits, (m, v), logits.dtype, "dlogits"), _matrix(dlogits, "dlogits")[2], _stream())
    if st:
        _check(st, "bz_distill_backward")
    return dlogits


# ------------------------------------------------------------------------- losses on one token a position

def _here(t: torch.Tensor, name: str, others=()):
    """The calls below launch on the current device's current stream: their tensors have to live there, `others` (None among them) too."""
    if not t.is_cuda:
        return
    here = torch._C._cuda_getDevice()
    if t.get_device() != here:
        raise ValueError("%s is on %s, the current device is cuda:%d: call under torch.cuda.device(%s.device)" % (name, t.device, here, name))
    for other in others:
        if other is not None and other.get_device() != here and other.is_cuda:
            raise ValueError("%s is on %s, another tensor of the call on %s" % (name, t.device, other.device))


def _row_tensor(t, shape, dtype, name: str):
    """(address, leading dimension) of a matrix of this shape and type."""
    if t.is_contiguous() and t.shape == shape and t.dtype is dtype and t.is_cuda:
        return t.data_ptr(), shape[1]
    return _shaped(t, shape, dtype, name), _matrix(t, name)[2]


def _token_operands(logits, index, dloss, dlogits, *others):
    """(m, arguments from logits to index, whether a gradient is wanted, dlogits, its address and leading dimension)."""
    m, v, ld = _matrix(logits, "logits")
    head = (logits.data_ptr(), ld, _dtype(logits, "logits"), m, v, _packed(index, (m,), torch.int32, "index"))
    _here(logits, "logits", (index, dloss, dlogits, *others))
    if dlogits is None:
        if dloss is None:
            return m, head, False, None, None, 0
        dlogits = _alike(logits)
        return m, head, True, dlogits, dlogits.data_ptr(), dlogits.stride(0) if m > 1 else v
    return m, head, True, dlogits, *_row_tensor(dlogits, logits.shape, logits.dtype, "dlogits")


def _made(t, like, shape, name):
    """(tensor, address) of a binary32 output; a new one if t is None."""
    if t is None:
        t = like.new_empty(shape) if like.dtype is torch.float32 else like.new_empty(shape, dtype=torch.float32)
        return t, t.data_ptr()
    return t, _packed(t, shape, torch.float32, name)


def _alike(t: torch.Tensor) -> torch.Tensor:
    """_like_rows() of a matrix, in one step where its rows are apart."""
    if t.is_contiguous():
        return torch.empty_like(t)
    m, n = t.shape
    ld = t.stride(0)
    return torch.empty_strided((m, n), (ld, 1), dtype=t.dtype, device=t.device) if m > 1 and n < ld <= 2 * n else t.new_empty((m, n))


def _new_rows(t: torch.Tensor, m: int, n: int):
    """(tensor, address, leading dimension): a new one like the matrix t, [m][n]."""
    new = _alike(t)
    return new, new.data_ptr(), new.stride(0) if m > 1 else n


def policy(logits: torch.Tensor, index: torch.Tensor, advantage: torch.Tensor, old_logp: torch.Tensor | None = None,
           ref_logp: torch.Tensor | None = None, kl: float = 0.0, clip_low: float = 0.2, clip_high: float = 0.2, temperature: float = 1.0,
           dloss: torch.Tensor | None = None, loss: torch.Tensor | None = None, logp: torch.Tensor | None = None,
           stats: torch.Tensor | None = None, dlogits: torch.Tensor | None = None):
    """bz_policy: the clipped policy loss of each position, with a KL term.  Returns (loss, logp, stats); with `dloss`
    (float32 [m]) or `dlogits` given also the gradient, from the same pass: (loss, logp, stats, dlogits)."""
    if logits.requires_grad:
        _unrecorded("policy", logits=logits)
    m, head, grad, dlogits, p_d, ld_d = _token_operands(logits, index, dloss, dlogits, advantage, old_logp, ref_logp, loss, logp, stats)
    p_advantage = _packed(advantage, (m,), torch.float32, "advantage")
    loss, p_loss = _made(loss, advantage, (m,), "loss")
    logp, p_logp = _made(logp, advantage, (m,), "logp")
    stats, p_stats = _made(stats, advantage, (m, 4), "stats")
    st = lib().bz_policy(*head, _packed(old_logp, (m,), torch.float32, "old_logp"), _packed(ref_logp, (m,), torch.float32, "ref_logp"),
                         p_advantage, temperature, clip_low, clip_high, kl,
                         _packed(dloss, (m,), torch.float32, "dloss"), p_loss, p_logp, p_stats, p_d, ld_d, _stream())
    if st:
        _check(st, "bz_policy")
    return (loss, logp, stats, dlogits) if grad else (loss, logp, stats)


def preference(logits: torch.Tensor, index: torch.Tensor, starts: torch.Tensor, ref_logp: torch.Tensor | None = None, beta: float = 0.1,
               margin: float = 0.0, smoothing: float = 0.0, mean: bool = False, temperature: float = 1.0,
               dloss: torch.Tensor | None = None, loss: torch.Tensor | None = None, reward: torch.Tensor | None = None,
               logp: torch.Tensor | None = None, stats: torch.Tensor | None = None, dlogits: torch.Tensor | None = None):
    """bz_preference: the paired preference loss of the sequences that `starts` (int32 [2 pairs + 1]) cuts the rows into, chosen
    ones first.  Returns (loss, reward, logp, stats); with `dloss` (float32 [pairs]) or `dlogits` given also the gradient:
    (loss, reward, logp, stats, dlogits)."""
    if logits.requires_grad:
        _unrecorded("preference", logits=logits)
    m, head, grad, dlogits, p_d, ld_d = _token_operands(logits, index, dloss, dlogits, starts, ref_logp, loss, reward, logp, stats)
    if starts.dim() != 1 or starts.shape[0] % 2 != 1:
        raise ValueError("starts must be [2 pairs + 1]")
    pairs = starts.shape[0] // 2
    loss, p_loss = _made(loss, logits, (pairs,), "loss")
    reward, p_reward = _made(reward, logits, (2 * pairs,), "reward")
    logp, p_logp = _made(logp, logits, (m,), "logp")
    stats, p_stats = _made(stats, logits, (m, 4), "stats")
    st = lib().bz_preference(*head, _packed(ref_logp, (m,), torch.float32, "ref_logp"), _packed(starts, starts.shape, torch.int32, "starts"), pairs,
                             temperature, beta, margin, smoothing, 1 if mean else 0, _packed(dloss, (pairs,), torch.float32, "dloss"), p_loss, p_reward,
                             p_logp, p_stats, p_d, ld_d, _stream())
    if st:
        _check(st, "bz_preference")
    return (loss, reward, logp, stats, dlogits) if grad else (loss, reward, logp, stats)


def token_loss_backward(logits: torch.Tensor, index: torch.Tensor, stats: torch.Tensor, dloss: torch.Tensor | None = None,
                        temperature: float = 1.0, dlogits: torch.Tensor | None = None) -> torch.Tensor:
    """bz_token_loss_backward: the gradient alone, with stats as policy() or preference() returned them; dloss as there (rows whose
    loss it does not hold get NaN)."""
    if dlogits is None:
        dlogits = _alike(logits)
    m, head, _, dlogits, p_d, ld_d = _token_operands(logits, index, dloss, dlogits, stats)
    if dloss is not None and dloss.dim() != 1:
        raise ValueError("dloss must be [m] or [pairs]")
    p_stats = _packed(stats, (m, 4), torch.float32, "stats")
    p_dloss, places = None, 0
    if dloss is not None:
        # a tensor without elements has no address, which would stand for ones
        p_dloss, places = _packed(dloss, dloss.shape, torch.float32, "dloss") or p_stats, dloss.shape[0]
    st = lib().bz_token_loss_backward(*head, temperature, p_stats, p_dloss, places, p_d, ld_d, _stream())
    if st:
        _check(st, "bz_token_loss_backward")
    return dlogits


# ------------------------------------------------------------------------- dropout, joins of blocks

def _collapsed(t: torch.Tensor, name: str):
    """(m, n, ld): the tensor as rows of one distance, in row-major order."""
    if t.is_contiguous():
        return 1, t.numel(), t.numel()
    dims = []      # from the last to the first: [size, stride]
    for size, stride in zip(reversed(t.shape), reversed(t.stride())):
        if size == 1:
            continue
        if dims and stride == dims[-1][0] * dims[-1][1]:
            dims[-1][0] *= size
        else:
            dims.append([size, stride])
    if dims[0][1] != 1:
        dims.insert(0, [1, 1])
    if len(dims) > 2 or (len(dims) == 2 and dims[1][1] < dims[0][0]):
        raise ValueError("%s must be rows of unit stride, one distance apart: make it contiguous" % name)
    (n, _), (m, ld) = dims if len(dims) == 2 else (dims[0], (1, dims[0][0]))
    return m, n, ld


def dropout(x: torch.Tensor, rate: float, rng: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """bz_dropout: x with the elements dropped that seed and offset in `rng` (int64 [2] on the device) name, the others scaled.  The
    gradient is the same call on the gradient.  `out` may be x itself."""
    if x.requires_grad:
        if torch.is_grad_enabled():
            raise ValueError("dropout: x requires a gradient, which this call does not record: call it under torch.no_grad() (or inside an "
                             "autograd.Function), and again on the gradient")
    dt = _dtype(x, "x")
    _here(x, "x", (rng, out))
    m, n, ld = _collapsed(x, "x")
    given = out
    if out is None:
        out = torch.empty_like(x) if m == 1 else x.new_empty(m, ld).as_strided(x.shape, x.stride()) if ld <= 2 * n else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if out.shape != x.shape or out.dtype != x.dtype or not out.is_cuda:
        raise ValueError("out must be a CUDA tensor like x")
    m2, n2, ld2 = _collapsed(out, "out")
    if m == 1 and m2 > 1:
        m, n, ld = m2, n2, n2
    elif m2 == 1:
        m2, n2, ld2 = m, n, n
    if n2 != n:
        raise ValueError("x and out must be cut into rows alike: make one of them contiguous")
    st = lib().bz_dropout(x.data_ptr(), ld, dt, m, n, rate, _packed(rng, (2,), torch.int64, "rng"), out.data_ptr(), ld2, _stream())
    if st:
        _check(st, "bz_dropout")
    _written(given)
    return out


def _written(*given):
    """The caller's tensors that a call has written, for who keeps one of them: torch counts only its own writes."""
    for t in given:
        if t is not None:
            torch._C._increment_version((t,))


_NORMS = {"rms": NORM_RMS, "layer": NORM_LAYER}


def _norm(name: str) -> int:
    try:
        return _NORMS[name]
    except KeyError:
        raise ValueError("norm must be rms or layer") from None


def _join_form(m, n, w_post, gate, w_pre, rate, rng):
    """Addresses of w_post, gate, its rows, rng, w_pre."""
    if gate is not None and (gate.dim() != 2 or gate.shape[1] != n or (m > 0 and gate.shape[0] == 0)):
        raise ValueError("gate must be [groups][%d], of one group at least" % n)
    if n == 0:
        gate = None      # it has no address, and rows without one are refused
    return (_packed(w_post, (n,), torch.float32, "w_post"), None if gate is None else _packed(gate, gate.shape, torch.float32, "gate"),
            0 if gate is None else gate.shape[0], _packed(rng, (2,), torch.int64, "rng"), _packed(w_pre, (n,), torch.float32, "w_pre"))


def join(x: torch.Tensor, y: torch.Tensor | None = None, w_post: torch.Tensor | None = None, gate: torch.Tensor | None = None,
         w_pre: torch.Tensor | None = None, norm: str = "rms", eps: float = 1e-6, residual_scale: float = 1.0, branch_scale: float = 1.0,
         rate: float = 0.0, rng: torch.Tensor | None = None, s: torch.Tensor | None = None, z: torch.Tensor | None = None,
         stats: torch.Tensor | None = None):
    """bz_join: s = residual_scale x + branch_scale gate drop(norm(y) w_post), z = norm(s) w_pre, for rows x, y [m][n] and weights
    float32 [n], gate float32 [groups][n].  Returns (s, z, stats); z is None without w_pre.  Without y: the norm alone, and s is
    written only if it is given (or residual_scale is not 1; otherwise the s that comes back is x).  For join_backward() stats keep x
    alive (itself, no copy of it), as automatic differentiation keeps what a backward pass reads."""
    if x.requires_grad or (y is not None and y.requires_grad):
        _unrecorded("join", x=x, y=y if y is not None else x)
    for name, w in (("w_post", w_post), ("gate", gate), ("w_pre", w_pre)):
        if w is not None and w.requires_grad:
            _unrecorded("join", **{name: w})
    m, n, ld_x = _matrix(x, "x")
    dt = _dtype(x, "x")
    _here(x, "x", (y, w_post, gate, w_pre, rng, s, z, stats))
    p_post, p_gate, groups, p_rng, p_pre = _join_form(m, n, w_post, gate, w_pre, rate, rng)
    p_y, ld_y = (None, 0) if y is None else _row_tensor(y, x.shape, x.dtype, "y")
    keep = s is None and y is None and residual_scale == 1.0 and w_pre is not None
    given = s, z
    p_s, ld_s, p_z, ld_z = None, 0, None, 0
    if s is not None:
        p_s, ld_s = _row_tensor(s, x.shape, x.dtype, "s")
    elif not keep:
        s, p_s, ld_s = _new_rows(x, m, n)
    if z is not None:
        p_z, ld_z = _row_tensor(z, x.shape, x.dtype, "z")
    elif w_pre is not None:
        z, p_z, ld_z = _new_rows(x, m, n)
    stats, p_stats = _made(stats, x, (m, 4), "stats")
    st = lib().bz_join(x.data_ptr(), ld_x, p_y, ld_y, dt, m, n, _norm(norm), eps, p_post, p_gate, groups, residual_scale, branch_scale, rate, p_rng,
                       p_pre, p_s, ld_s, p_z, ld_z, p_stats, _stream())
    if st:
        _check(st, "bz_join")
    _written(*given)
    p_x = x.data_ptr()
    try:
        version = x._version
    except RuntimeError:      # a tensor of inference mode counts no writes
        version = None
    stats._stream_in = x, version, p_x != 0 and (p_s == p_x or p_z == p_x)
    return x if keep else s, z, stats


def _stream_in(stream: torch.Tensor, stats: torch.Tensor) -> torch.Tensor:
    """The x of the join() call that stats come from, where they keep it; `stream` may be that x or the s of the call."""
    x, version, over = getattr(stats, "_stream_in", (stream, None, False))
    if x is stream and not over:
        return x
    if stream.shape != x.shape or stream.dtype is not x.dtype or stream.device != x.device:
        raise ValueError("join_backward: the stream must be like the x that join() had")
    there = stream.data_ptr() == x.data_ptr()
    if over and there:
        raise ValueError("join_backward: join() has written over its x, which the gradient needs: keep a copy and give it as x=")
    if over or there:
        return stream
    if version is not None and x._version != version:
        raise ValueError("join_backward: the x that join() had was written since: give the stream as it went in as x=")
    return x


def join_workspace_bytes(m: int, n: int, groups: int = 0) -> int:
    return int(lib().bz_join_workspace_bytes(m, n, groups))


def join_backward(stream: torch.Tensor | None = None, y: torch.Tensor | None = None, stats: torch.Tensor | None = None, ds: torch.Tensor | None = None,
                  dz: torch.Tensor | None = None, w_post: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                  w_pre: torch.Tensor | None = None, norm: str = "rms", residual_scale: float = 1.0, branch_scale: float = 1.0,
                  rate: float = 0.0, rng: torch.Tensor | None = None, dx: torch.Tensor | None = None, dy: torch.Tensor | None = None,
                  dw_post: torch.Tensor | None = None, dgate: torch.Tensor | None = None, dw_pre: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None, x: torch.Tensor | None = None):
    """bz_join_backward, with y and stats as join() had and returned them: returns (dx, dy, dw_post, dgate, dw_pre), None for what the call has
    no operand of.  `stream` is the x that went into join() or the s that came out: the gradient is formed from x, which stats keep.  A copy of
    stats keeps none, and `stream` is x then; x=... is taken as it is.  dw_post, dgate and dw_pre may be views of a gradient row."""
    if stats is None or (x is None) == (stream is None):
        raise TypeError("join_backward needs stats and either a stream or x")
    if x is None:
        x = _stream_in(stream, stats)
    m, n, ld = _matrix(x, "x")
    dt = _dtype(x, "x")
    _here(x, "x", (y, stats, ds, dz, w_post, gate, w_pre, rng, dx, dy, dw_post, dgate, dw_pre, workspace))
    p_post, p_gate, groups, p_rng, p_pre = _join_form(m, n, w_post, gate, w_pre, rate, rng)
    like = x.shape, x.dtype
    given = dx, dy
    p_y, ld_y = (None, 0) if y is None else _row_tensor(y, *like, "y")
    p_ds, ld_ds = (None, 0) if ds is None else _row_tensor(ds, *like, "ds")
    p_dz, ld_dz = (None, 0) if dz is None else _row_tensor(dz, *like, "dz")
    dx, p_dx, ld_dx = (dx, *_row_tensor(dx, *like, "dx")) if dx is not None else _new_rows(x, m, n)
    p_dy, ld_dy = None, 0
    if dy is not None:
        p_dy, ld_dy = _row_tensor(dy, *like, "dy")
    elif y is not None:
        dy, p_dy, ld_dy = _new_rows(y, m, n)
    p_dpost = p_dgate = p_dpre = None
    if w_post is not None:
        dw_post, p_dpost = _made(dw_post, x, (n,), "dw_post")
    if gate is not None:
        dgate, p_dgate = _made(dgate, x, gate.shape, "dgate")
    if w_pre is not None:
        dw_pre, p_dpre = _made(dw_pre, x, (n,), "dw_pre")
    room = (None, 0)
    if workspace is not None:
        room = _room(workspace)
    elif w_post is not None or gate is not None or w_pre is not None:
        size = max(256, lib().bz_join_workspace_bytes(m, n, groups))
        workspace = x.new_empty(size, dtype=torch.uint8)
        room = workspace.data_ptr(), size
    st = lib().bz_join_backward(x.data_ptr(), ld, p_y, ld_y, dt, m, n, _norm(norm), p_post, p_gate, groups, residual_scale, branch_scale, rate, p_rng,
                                p_pre, _packed(stats, (m, 4), torch.float32, "stats"), p_ds, ld_ds, p_dz, ld_dz, p_dx, ld_dx, p_dy, ld_dy,
                                p_dpost, p_dgate, p_dpre, *room, _stream())
    if st:
        _check(st, "bz_join_backward")
    _written(*given)
    return dx, dy, dw_post, dgate, dw_pre
