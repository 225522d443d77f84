"""Thin binding over libdeft.so (ctypes): the same names as the C ABI, argument marshalling only.

Host tables are numpy arrays, device buffers are torch CUDA tensors (used for memory and
streams only).  Nothing here computes anything of the method, and there is no fallback:
if the CUDA library is missing or fails to load, importing a device call raises.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Tuple

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdeft.so")

OK = 0
WARN_K_INEXACT = 1
ERR_INVALID_ARG = -1
ERR_INFEASIBLE_K = -2
ERR_NONFINITE_NORM = -3
ERR_CAPACITY = -4
ERR_CUDA = -5
ERR_TOO_LARGE = -6
MODE_PAPER = 0
MODE_EXACT = 1


class DeftError(RuntimeError):
    def __init__(self, call: str, status: int, detail: str = ""):
        self.status = status
        super().__init__("%s failed: %s%s" % (call, status_string(status), detail))


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libdeft.so from the package directory.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                "libdeft.so is missing at %s: build it with `python -m paper_2307_03500_b200.build` "
                "(there is no CPU fallback)" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        c = ctypes
        vp, i32, i64, sz = c.c_void_p, c.c_int32, c.c_int64, c.c_size_t
        L.deft_status_string.restype = c.c_char_p
        L.deft_status_string.argtypes = [i32]
        L.deft_last_cuda_error.restype = i32
        L.deft_last_cuda_error.argtypes = []
        L.deft_debug_select_timing.restype = None
        L.deft_debug_select_timing.argtypes = [vp]
        L.deft_debug_select_kernel.restype = None
        L.deft_debug_select_kernel.argtypes = [i32]
        L.deft_debug_select_ring.restype = None
        L.deft_debug_select_ring.argtypes = [i32]
        L.deft_debug_step_staging.restype = None
        L.deft_debug_step_staging.argtypes = [i32]
        L.deft_select_stats.restype = i32
        L.deft_select_stats.argtypes = [vp, sz, i32, vp, vp]
        L.deft_select_launch_max_elems.restype = i64
        L.deft_select_launch_max_elems.argtypes = []
        L.deft_split_layers.restype = i32
        L.deft_split_layers.argtypes = [vp, i32, i32, vp, vp, i32, vp]
        L.deft_allocate_k.restype = i32
        L.deft_allocate_k.argtypes = [vp, vp, i32, i64, i32, vp, vp]
        L.deft_partition.restype = i32
        L.deft_partition.argtypes = [vp, vp, i32, i32, vp, vp]
        L.deft_rank_bin.restype = i32
        L.deft_rank_bin.argtypes = [i64, i32, i32]
        L.deft_bin_layers.restype = i32
        L.deft_bin_layers.argtypes = [vp, i32, i32, vp, i32, vp]
        L.deft_workspace_bytes.restype = sz
        L.deft_workspace_bytes.argtypes = [i64, i32]
        L.deft_layer_norms.restype = i32
        L.deft_layer_norms.argtypes = [vp, vp, i64, vp, i32, vp, vp, sz, vp]
        L.deft_layer_norms_static_max_slots.restype = i64
        L.deft_layer_norms_static_max_slots.argtypes = []
        L.deft_layer_norms_static.restype = i32
        L.deft_layer_norms_static.argtypes = [vp, vp, i64, vp, i32, vp, vp]
        L.deft_select.restype = i32
        L.deft_select.argtypes = [vp, vp, vp, vp, i32, vp, vp, i64, vp, sz, vp]
        L.deft_plan_bytes.restype = sz
        L.deft_plan_bytes.argtypes = [i32, i32]
        L.deft_plan_build.restype = i32
        L.deft_plan_build.argtypes = [vp, vp, vp, i32, i32, i64, vp, sz]
        L.deft_plan_rank_info.restype = i32
        L.deft_plan_rank_info.argtypes = [vp, i32, vp, vp, vp, vp]
        L.deft_plan_rank_table.restype = i32
        L.deft_plan_rank_table.argtypes = [vp, i32, vp, vp, vp, vp]
        L.deft_step.restype = i32
        L.deft_step.argtypes = [vp, vp, i64, vp, vp, i32, i32, i64, i32, i32, i64, i32, vp, vp, vp, vp, vp, vp, vp, sz,
                                vp, vp, vp, i64, vp, sz, vp, vp]
        f64, u64 = c.c_double, c.c_uint64
        L.deft_layer_norms_part.restype = i32
        L.deft_layer_norms_part.argtypes = [vp, vp, i64, vp, i32, vp, i32, vp, vp, sz, vp]
        L.deft_step_part.restype = i32
        L.deft_step_part.argtypes = L.deft_step.argtypes[:3] + [vp, i32] + L.deft_step.argtypes[3:]
        L.deft_embed.restype = i32
        L.deft_embed.argtypes = [vp, i32, i64, i64, i64, vp, i32, i64, f64, vp, i64, i64, f64, u64, u64, vp, vp, i32, i64, vp]
        L.deft_embed_workspace_bytes.restype = sz
        L.deft_embed_workspace_bytes.argtypes = [i64, i64, i64]
        L.deft_embed_grad.restype = i32
        L.deft_embed_grad.argtypes = [vp, i32, i64, vp, i32, i64, i64, i64, i64, f64, f64, u64, u64, vp, vp, i32, vp, sz, vp]
        L.deft_dropout.restype = i32
        L.deft_dropout.argtypes = [vp, i32, i64, vp, i64, vp, i32, i64, i64, i64, f64, u64, u64, vp, vp]
        L.deft_layer_norm.restype = i32
        L.deft_layer_norm.argtypes = [vp, i32, i64, vp, i64, vp, i64, vp, vp, i32, vp, i32, i64, i64, i64, f64, vp, vp, vp]
        L.deft_layer_norm_workspace_bytes.restype = sz
        L.deft_layer_norm_workspace_bytes.argtypes = [i64, i64]
        L.deft_layer_norm_grad.restype = i32
        L.deft_layer_norm_grad.argtypes = [vp, i32, i64, vp, i32, i64, vp, vp, vp, i32, vp, i64, vp, i64, vp, vp, i64, i64, i32, f64, vp, sz, vp]
        L.deft_rotary_frequencies.restype = i32
        L.deft_rotary_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, vp]
        L.deft_rotary.restype = i32
        L.deft_rotary.argtypes = [vp, vp, vp, vp, i32, i64, i64, i64, i64, vp, i64, i32, i32, f64, vp, i32, vp]
        L.deft_distill.restype = i32
        L.deft_distill.argtypes = [vp, i32, i64, i64, i64, vp, i32, i64, vp, i32, i64, i64, vp, f64, vp, f64, vp, vp, i64, vp]
        L.deft_workspace_init.restype = i32
        L.deft_workspace_init.argtypes = [vp, sz, i32, vp]
        L.deft_threshold_select.restype = i32
        L.deft_threshold_select.argtypes = [vp, i64, ctypes.c_float, i32, vp, vp, i64, vp, vp, sz, vp]
        L.deft_clt_leader.restype = i32
        L.deft_clt_leader.argtypes = [i64, i32]
        L.deft_gather_update.restype = i32
        L.deft_gather_update.argtypes = [vp, i64, vp, i64, vp, vp]
        L.deft_plan_step.restype = i32
        L.deft_plan_step.argtypes = [vp, vp, i32, i32, i64, i32, i32, i64, vp, vp, vp, vp, vp, sz, vp, vp, sz, vp]
        L.deft_partition_model.restype = i32
        L.deft_partition_model.argtypes = [vp, vp, i32, i32, i32, vp, vp]
        L.deft_plan_upload.restype = i32
        L.deft_plan_upload.argtypes = [vp, vp, vp, sz, vp]
        L.deft_select_planned.restype = i32
        L.deft_select_planned.argtypes = [vp, vp, vp, i32, vp, vp, i64, vp, sz, vp]
        L.deft_select_update_all.restype = i32
        L.deft_select_update_all.argtypes = [vp, i64, vp, vp, vp, vp, i64, vp, sz, vp]
        L.deft_select_update_ranks.restype = i32
        L.deft_select_update_ranks.argtypes = [vp, i64, vp, vp, i32, i32, vp, vp, i64, vp, sz, vp, vp]
        L.deft_error_eq2.restype = i32
        L.deft_error_eq2.argtypes = [vp, i32, vp]
        L.deft_union_workspace_bytes.restype = sz
        L.deft_union_workspace_bytes.argtypes = [i64]
        L.deft_index_union.restype = i32
        L.deft_index_union.argtypes = [vp, i64, i64, vp, i64, vp, vp, sz, vp]
        L.deft_sum_into.restype = i32
        L.deft_sum_into.argtypes = [vp, vp, i64, vp]
        L.deft_average.restype = i32
        L.deft_average.argtypes = [vp, i64, i32, vp]
        L.deft_vector_norm_workspace_bytes.restype = sz
        L.deft_vector_norm_workspace_bytes.argtypes = [i64]
        L.deft_vector_norm.restype = i32
        L.deft_vector_norm.argtypes = [vp, i64, vp, vp, sz, vp]
        L.deft_residual_update.restype = i32
        L.deft_residual_update.argtypes = [vp, i64, vp, i64, vp]
        L.deft_topk_baseline.restype = i32
        L.deft_topk_baseline.argtypes = [vp, i64, i64, vp, vp, vp, sz, vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().deft_status_string(int(status)).decode()


def _check(call: str, status: int, allow_warn: bool = False) -> int:
    if status < 0 or (status > 0 and not allow_warn):
        detail = ""
        if status == ERR_CUDA:
            detail = " (cudaError %d)" % lib().deft_last_cuda_error()
        raise DeftError(call, status, detail)
    return status


def _np(a, dtype) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=dtype)


def _hp(a: Optional[np.ndarray]):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


def _dp(t, dtype=None):
    """Device pointer of a contiguous CUDA tensor."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError("expected dtype %s, got %s" % (dtype, t.dtype))
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    """The handle of `stream`, or of the current stream."""
    if stream is None:   # (the handle alone: a Stream object takes 3 us to build, as long as a launch)
        import torch
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


# ------------------------------------------------------------------------------------------
# host planners
# ------------------------------------------------------------------------------------------
def deft_split_layers(tensor_sizes, n_workers: int) -> Tuple[np.ndarray, np.ndarray]:
    """Algorithm 2 -> (layer_start int64[L+1], layer_tensor int32[L])."""
    sizes = _np(tensor_sizes, np.int64)
    L = ctypes.c_int32(0)
    st = lib().deft_split_layers(_hp(sizes), sizes.size, int(n_workers), _hp(np.zeros(1, np.int64)), None, 0,
                                 ctypes.byref(L))
    if st != ERR_CAPACITY:
        _check("deft_split_layers", st)
    cap = int(L.value)
    start = np.zeros(cap + 1, dtype=np.int64)
    tensor = np.zeros(cap, dtype=np.int32)
    _check("deft_split_layers",
           lib().deft_split_layers(_hp(sizes), sizes.size, int(n_workers), _hp(start), _hp(tensor), cap,
                                   ctypes.byref(L)))
    return start, tensor


def deft_allocate_k(norms, layer_size, k: int, mode: int = MODE_EXACT) -> Tuple[np.ndarray, int, int]:
    """Algorithm 3 -> (k_l int64[L], sum_k, status) ; status may be WARN_K_INEXACT in PAPER mode."""
    nr = _np(norms, np.float64)
    sz = _np(layer_size, np.int64)
    if nr.size != sz.size:
        raise ValueError("norms and layer_size differ in length")
    k_l = np.zeros(sz.size, dtype=np.int64)
    s = ctypes.c_int64(0)
    st = _check("deft_allocate_k",
                lib().deft_allocate_k(_hp(nr), _hp(sz), sz.size, int(k), int(mode), _hp(k_l), ctypes.byref(s)),
                allow_warn=True)
    return k_l, int(s.value), st


COST_EQ3 = 0
COST_SIZE = 1


def deft_partition_model(layer_size, k_l, n_workers: int, cost_model: int) -> Tuple[np.ndarray, np.ndarray]:
    """Algorithm 4's packing under a load model (COST_EQ3 / COST_SIZE) -> (bins int32[L], loads float64[N])."""
    sz = _np(layer_size, np.int64)
    kl = None if k_l is None else _np(k_l, np.int64)
    if kl is not None and kl.size != sz.size:
        raise ValueError("k_l and layer_size differ in length")
    bins = np.zeros(sz.size, dtype=np.int32)
    load = np.zeros(int(n_workers), dtype=np.float64)
    _check("deft_partition_model", lib().deft_partition_model(_hp(sz), _hp(kl), sz.size, int(n_workers),
                                                              int(cost_model), _hp(bins), _hp(load)))
    return bins, load


def deft_partition(layer_size, k_l, n_workers: int) -> Tuple[np.ndarray, np.ndarray]:
    """Algorithm 4 packing -> (bin_of_layer int32[L], bin_load float64[N])."""
    sz = _np(layer_size, np.int64)
    kl = _np(k_l, np.int64)
    if kl.size != sz.size:
        raise ValueError("k_l and layer_size differ in length")
    bins = np.zeros(sz.size, dtype=np.int32)
    load = np.zeros(int(n_workers), dtype=np.float64)
    _check("deft_partition", lib().deft_partition(_hp(sz), _hp(kl), sz.size, int(n_workers), _hp(bins), _hp(load)))
    return bins, load


def deft_rank_bin(iteration: int, rank: int, n_workers: int) -> int:
    b = lib().deft_rank_bin(int(iteration), int(rank), int(n_workers))
    if b < 0:
        raise DeftError("deft_rank_bin", ERR_INVALID_ARG)
    return int(b)


def deft_bin_layers(bin_of_layer, bin_id: int) -> np.ndarray:
    bins = _np(bin_of_layer, np.int32)
    out = np.zeros(bins.size, dtype=np.int32)
    n = ctypes.c_int32(0)
    _check("deft_bin_layers", lib().deft_bin_layers(_hp(bins), bins.size, int(bin_id), _hp(out), out.size,
                                                    ctypes.byref(n)))
    return out[: n.value].copy()


# ------------------------------------------------------------------------------------------
# device calls
# ------------------------------------------------------------------------------------------
def deft_workspace_bytes(max_elems: int, max_layers: int) -> int:
    return int(lib().deft_workspace_bytes(int(max_elems), int(max_layers)))


def alloc_workspace(max_elems: int, max_layers: int, device="cuda"):
    """A torch uint8 tensor of deft_workspace_bytes() bytes (torch allocations are 512-byte aligned)."""
    import torch
    ws = torch.empty(deft_workspace_bytes(max_elems, max_layers), dtype=torch.uint8, device=device)
    with torch.cuda.device(ws.device):
        _check("deft_workspace_init", lib().deft_workspace_init(_dp(ws), ws.numel(), int(max_layers), _stream(None)))
    return ws


def deft_layer_norms(resid_acc, grad, layer_start_d, norms_d, ws, stream=None) -> None:
    import torch
    n_g = resid_acc.numel()
    L = layer_start_d.numel() - 1
    if grad is not None and grad.numel() != n_g:
        raise ValueError("grad and resid_acc differ in length")
    if norms_d.numel() < L:
        raise ValueError("norms_d too small")
    _check("deft_layer_norms",
           lib().deft_layer_norms(_dp(resid_acc, torch.float32), _dp(grad, torch.float32), n_g,
                                  _dp(layer_start_d, torch.int64), L, _dp(norms_d, torch.float64),
                                  _dp(ws), ws.numel() * ws.element_size(), _stream(stream)))


def _parts(parts):
    """(begin, end) pairs as a host array for the library, and their number."""
    n = len(parts)
    if any(len(part) != 2 for part in parts):
        raise ValueError("parts: (begin, end) pairs")
    return (ctypes.c_int64 * max(1, 2 * n))(*[int(x) for part in parts for x in part]), n


def deft_layer_norms_part(resid_acc, grad, parts, layer_start_d, norms_d, ws, stream=None) -> None:
    """deft_layer_norms of a vector whose parts [(begin, end), ...] hold their gradient already, on the tensors' device."""
    import torch
    n_g = resid_acc.numel()
    L = layer_start_d.numel() - 1
    if grad is not None and grad.numel() != n_g:
        raise ValueError("grad and resid_acc differ in length")
    if norms_d.numel() < L:
        raise ValueError("norms_d too small")
    pt, n_parts = _parts(parts)
    _call("deft_layer_norms_part", _device(resid_acc, grad, layer_start_d, norms_d, ws), stream,
          _dp(resid_acc, torch.float32), _dp(grad, torch.float32), n_g, pt, n_parts, _dp(layer_start_d, torch.int64), L,
          _dp(norms_d, torch.float64), _dp(ws), ws.numel() * ws.element_size())


def deft_layer_norms_static(resid_acc, grad, layer_start_d, norms_d, stream=None) -> None:
    """deft_layer_norms without a workspace, for callers that may not allocate device memory: the scratch is a
    fixed array inside the library (limit: ceil(n_g/8192) + L + 1 <= deft_layer_norms_static_max_slots())."""
    import torch
    n_g = resid_acc.numel()
    L = layer_start_d.numel() - 1
    if grad is not None and grad.numel() != n_g:
        raise ValueError("grad and resid_acc differ in length")
    if norms_d.numel() < L:
        raise ValueError("norms_d too small")
    _check("deft_layer_norms_static",
           lib().deft_layer_norms_static(_dp(resid_acc, torch.float32), _dp(grad, torch.float32), n_g,
                                         _dp(layer_start_d, torch.int64), L, _dp(norms_d, torch.float64),
                                         _stream(stream)))


def deft_select(acc, layer_start_h, k_l_h, my_layers_h, val_d, idx_d, ws, stream=None) -> int:
    """Algorithm 5 for one rank.  Returns the number of entries written (sum of k_l over my layers)."""
    import torch
    ls = _np(layer_start_h, np.int64)
    kl = _np(k_l_h, np.int64)
    my = _np(my_layers_h, np.int32)
    if kl.size != ls.size - 1:
        raise ValueError("k_l_h and layer_start_h disagree")
    if my.size and (my.min() < 0 or my.max() >= kl.size):
        raise ValueError("layer id out of range")
    cap = min(val_d.numel(), idx_d.numel())
    _check("deft_select",
           lib().deft_select(_dp(acc, torch.float32), _hp(ls), _hp(kl), _hp(my), my.size,
                             _dp(val_d, torch.float32), _dp(idx_d, torch.int64), cap, _dp(ws),
                             ws.numel() * ws.element_size(), _stream(stream)))
    return int(kl[my].sum()) if my.size else 0


def deft_debug_select_timing(timing_d) -> None:
    """Diagnostic phase stamps of the selection kernel: a zeroed CUDA uint64/int64 tensor of 1024, or None."""
    lib().deft_debug_select_timing(None if timing_d is None else _dp(timing_d))


def deft_debug_select_kernel(single_pass) -> None:
    """True / False: force the single-pass / the five-step selection kernel; None: by call size (default)."""
    lib().deft_debug_select_kernel(-1 if single_pass is None else (1 if single_pass else 0))


def deft_debug_select_ring(on: bool) -> None:
    """The single-pass kernel reads through a ring of bulk copies (True, the default) or with plain loads (False)."""
    lib().deft_debug_select_ring(1 if on else 0)


def deft_debug_step_staging(on: bool) -> None:
    """deft_step for all workers stages during the accumulate pass (True, the default) or leaves the read to the
    selection launch (False)."""
    lib().deft_debug_step_staging(1 if on else 0)


def deft_select_stats(ws, n_layers: int, stream=None) -> dict:
    out = np.zeros(8, dtype=np.uint64)
    _check("deft_select_stats", lib().deft_select_stats(_dp(ws), ws.numel() * ws.element_size(), n_layers,
                                                        _hp(out), _stream(stream)))
    return {"one_read": int(out[0]), "cut_failed": int(out[1]), "no_cut": int(out[2]), "ring_gave_up": int(out[3]), "staged_entries": int(out[4])}


def deft_select_launch_max_elems() -> int:
    return int(lib().deft_select_launch_max_elems())


def deft_plan_bytes(n_layers: int, n_workers: int) -> int:
    return int(lib().deft_plan_bytes(int(n_layers), int(n_workers)))


def deft_plan_build(layer_start_h, k_l_h, bin_of_layer_h, n_workers: int, iteration: int,
                    out: Optional[np.ndarray] = None) -> np.ndarray:
    """Builds the step's plan blob on the host.  ``out`` may be a uint8 numpy view of pinned memory."""
    ls = _np(layer_start_h, np.int64)
    kl = _np(k_l_h, np.int64)
    bins = _np(bin_of_layer_h, np.int32)
    L = kl.size
    if ls.size != L + 1 or bins.size != L:
        raise ValueError("layer_start_h, k_l_h and bin_of_layer_h disagree")
    need = deft_plan_bytes(L, n_workers)
    if need == 0:
        raise DeftError("deft_plan_bytes", ERR_INVALID_ARG)
    if out is None:
        out = np.empty(need, dtype=np.uint8)
    if out.dtype != np.uint8 or not out.flags.c_contiguous or out.size < need:
        raise ValueError("plan buffer must be contiguous uint8 of at least %d bytes" % need)
    _check("deft_plan_build", lib().deft_plan_build(_hp(ls), _hp(kl), _hp(bins), L, int(n_workers), int(iteration),
                                                    _hp(out), out.size))
    return out


def deft_plan_rank_info(plan_h: np.ndarray, rank: int) -> Tuple[int, int, int, int]:
    """(layers, elements scanned, entries selected, sum of k over lower ranks) of one rank."""
    n = ctypes.c_int32(0)
    e, k, o = ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_int64(0)
    _check("deft_plan_rank_info", lib().deft_plan_rank_info(_hp(plan_h), int(rank), ctypes.byref(n), ctypes.byref(e),
                                                            ctypes.byref(k), ctypes.byref(o)))
    return int(n.value), int(e.value), int(k.value), int(o.value)


def deft_plan_rank_table(plan_h: np.ndarray, n_workers: int):
    """(layers int32[N], elements int64[N], entries int64[N], output offsets int64[N]) of all ranks."""
    n = np.zeros(n_workers, dtype=np.int32)
    e = np.zeros(n_workers, dtype=np.int64)
    k = np.zeros(n_workers, dtype=np.int64)
    o = np.zeros(n_workers, dtype=np.int64)
    _check("deft_plan_rank_table", lib().deft_plan_rank_table(_hp(plan_h), int(n_workers), _hp(n), _hp(e), _hp(k),
                                                              _hp(o)))
    return n, e, k, o


def deft_plan_upload(plan_h: np.ndarray, plan_d, ws, stream=None) -> None:
    if plan_d.numel() * plan_d.element_size() < plan_h.size:
        raise ValueError("plan_d smaller than the plan")
    _check("deft_plan_upload", lib().deft_plan_upload(_hp(plan_h), _dp(plan_d), _dp(ws),
                                                      ws.numel() * ws.element_size(), _stream(stream)))


def deft_plan_step(norms, layer_start_h, n_workers: int, k: int, mode: int, iteration: int, plan_h: np.ndarray,
                   plan_d, ws, stream=None, cost_model: int = 0):
    """Algorithm 3 + Algorithm 4 + plan build + plan upload in one call.
    Returns (k_l int64[L], sum_k, bin_of_layer int32[L], bin_load float64[N], status)."""
    nr = _np(norms, np.float64)
    ls = _np(layer_start_h, np.int64)
    L = nr.size
    if ls.size != L + 1:
        raise ValueError("norms and layer_start_h disagree")
    if plan_d.numel() * plan_d.element_size() < deft_plan_bytes(L, n_workers) or plan_h.dtype != np.uint8 or \
            not plan_h.flags.c_contiguous:
        raise ValueError("plan buffers too small or not contiguous uint8")
    k_l = np.empty(L, dtype=np.int64)
    bins = np.empty(L, dtype=np.int32)
    load = np.empty(int(n_workers), dtype=np.float64)
    s = ctypes.c_int64(0)
    st = _check("deft_plan_step",
                lib().deft_plan_step(_hp(nr), _hp(ls), L, int(n_workers), int(k), int(mode), int(cost_model),
                                     int(iteration), _hp(k_l),
                                     ctypes.byref(s), _hp(bins), _hp(load), _hp(plan_h), plan_h.size, _dp(plan_d),
                                     _dp(ws), ws.numel() * ws.element_size(), _stream(stream)),
                allow_warn=True)
    return k_l, int(s.value), bins, load, st


def deft_step(resid_acc, grad, layer_start_h, layer_start_d, n_workers: int, k: int, mode: int, cost_model: int,
              iteration: int, rank: int, norms_d, norms_h_pinned, k_l_out: np.ndarray, bins_out: np.ndarray,
              load_out: np.ndarray, plan_h: np.ndarray, plan_d, val_d, idx_d, ws, events=None, stream=None):
    """One whole step in one C call (rank = -1: all workers in one launch).  The output arrays
    (k_l_out int64[L], bins_out int32[L], load_out float64[N]) are filled in place.
    norms_h_pinned: a (pinned) torch float64 CPU tensor of L.  events: optional 4 torch CUDA events.
    Returns (sum_k, status)."""
    import torch
    ls = _np(layer_start_h, np.int64)
    L = ls.size - 1
    ev = None
    if events is not None:
        flat = []
        for e in events:
            if e.cuda_event == 0:   # torch creates the handle lazily, on first record
                e.record()
            flat.append(e.cuda_event)
        ev = (ctypes.c_void_p * 4)(*flat)
    s = ctypes.c_int64(0)
    st = _check("deft_step",
                lib().deft_step(_dp(resid_acc, torch.float32), None if grad is None else _dp(grad, torch.float32),
                                resid_acc.numel(), _hp(ls), _dp(layer_start_d, torch.int64), L, int(n_workers), int(k),
                                int(mode), int(cost_model), int(iteration), int(rank), _dp(norms_d, torch.float64),
                                ctypes.c_void_p(norms_h_pinned.data_ptr()), _hp(k_l_out), ctypes.byref(s),
                                _hp(bins_out), _hp(load_out), _hp(plan_h), plan_h.size, _dp(plan_d),
                                _dp(val_d, torch.float32), _dp(idx_d, torch.int64), min(val_d.numel(), idx_d.numel()),
                                _dp(ws), ws.numel() * ws.element_size(), ev, _stream(stream)),
                allow_warn=True)
    return int(s.value), st


def deft_select_planned(acc, plan_h: np.ndarray, plan_d, rank: int, val_d, idx_d, ws, stream=None) -> None:
    """Algorithm 5 for one rank of an uploaded plan (one kernel launch)."""
    import torch
    cap = min(val_d.numel(), idx_d.numel())
    _check("deft_select_planned",
           lib().deft_select_planned(_dp(acc, torch.float32), _hp(plan_h), _dp(plan_d), int(rank),
                                     _dp(val_d, torch.float32) if cap else None,
                                     _dp(idx_d, torch.int64) if cap else None, cap, _dp(ws),
                                     ws.numel() * ws.element_size(), _stream(stream)))


def deft_select_update_ranks(acc, plan_h: np.ndarray, plan_d, rank_begin: int, rank_end: int, val_d, idx_d, ws,
                             events=None, stream=None) -> None:
    """Selection + residual update for a range of simulated ranks (one C call).
    events: optional list of (before, between, after) torch.cuda.Event triples, one per rank."""
    import torch
    ev = None
    if events is not None:
        if len(events) != rank_end - rank_begin:
            raise ValueError("one event triple per rank expected")
        flat = []
        for tri in events:
            for e in tri:
                if e.cuda_event == 0:   # torch creates the handle lazily, on first record
                    e.record()
                flat.append(e.cuda_event)
        ev = (ctypes.c_void_p * len(flat))(*flat)
    _check("deft_select_update_ranks",
           lib().deft_select_update_ranks(_dp(acc, torch.float32), acc.numel(), _hp(plan_h), _dp(plan_d),
                                          int(rank_begin), int(rank_end), _dp(val_d, torch.float32),
                                          _dp(idx_d, torch.int64), min(val_d.numel(), idx_d.numel()), _dp(ws),
                                          ws.numel() * ws.element_size(), ev, _stream(stream)))


def deft_select_update_all(acc, plan_h: np.ndarray, plan_d, val_d, idx_d, ws, stream=None) -> None:
    """Selection + residual update for ALL simulated ranks of the plan in one launch."""
    import torch
    _check("deft_select_update_all",
           lib().deft_select_update_all(_dp(acc, torch.float32), acc.numel(), _hp(plan_h), _dp(plan_d),
                                        _dp(val_d, torch.float32), _dp(idx_d, torch.int64),
                                        min(val_d.numel(), idx_d.numel()), _dp(ws), ws.numel() * ws.element_size(),
                                        _stream(stream)))


def deft_threshold_select(acc, threshold: float, val_d, idx_d, count_d, ws, zero_selected: bool = False,
                          stream=None) -> None:
    """Hard-threshold sparsifier (Section 3.2): entries with magnitude > threshold, ascending index.
    count_d: CUDA int64 tensor of one element that receives the total count."""
    import torch
    cap = 0 if val_d is None or idx_d is None else min(val_d.numel(), idx_d.numel())
    _check("deft_threshold_select",
           lib().deft_threshold_select(_dp(acc, torch.float32), acc.numel(), float(threshold), int(bool(zero_selected)),
                                       _dp(val_d, torch.float32) if cap else None,
                                       _dp(idx_d, torch.int64) if cap else None, cap, _dp(count_d, torch.int64),
                                       _dp(ws), ws.numel() * ws.element_size(), _stream(stream)))


def deft_clt_leader(iteration: int, n_workers: int) -> int:
    r = int(lib().deft_clt_leader(int(iteration), int(n_workers)))
    if r < 0:
        raise DeftError("deft_clt_leader", ERR_INVALID_ARG)
    return r


def deft_gather_update(acc, idx_d, count: int, val_d, stream=None) -> None:
    """CLT-k follower: val_d[i] = acc[idx_d[i]], then that entry is cleared."""
    import torch
    if count > idx_d.numel() or count > val_d.numel():
        raise ValueError("count exceeds idx_d / val_d")
    _check("deft_gather_update",
           lib().deft_gather_update(_dp(acc, torch.float32), acc.numel(), _dp(idx_d, torch.int64), int(count),
                                    _dp(val_d, torch.float32), _stream(stream)))


def deft_error_eq2(worker_errors) -> float:
    w = _np(worker_errors, np.float64)
    out = np.zeros(1, dtype=np.float64)
    _check("deft_error_eq2", lib().deft_error_eq2(_hp(w), int(w.size), _hp(out)))
    return float(out[0])


def deft_union_workspace_bytes(n_g: int) -> int:
    return int(lib().deft_union_workspace_bytes(int(n_g)))


def deft_index_union(idx_d, count: int, n_g: int, union_d, count_d, ws, stream=None) -> None:
    """Sorted set of idx_d[:count] into union_d (as many as fit), its size into count_d (device int64)."""
    _check("deft_index_union", lib().deft_index_union(_dp(idx_d), int(count), int(n_g), _dp(union_d),
                                                      union_d.numel() if union_d is not None else 0, _dp(count_d),
                                                      _dp(ws), ws.numel() * ws.element_size(), _stream(stream)))


def deft_sum_into(dst, src, count: int, stream=None) -> None:
    _check("deft_sum_into", lib().deft_sum_into(_dp(dst), _dp(src), int(count), _stream(stream)))


def deft_average(sum_d, count: int, n_workers: int, stream=None) -> None:
    _check("deft_average", lib().deft_average(_dp(sum_d), int(count), int(n_workers), _stream(stream)))


def deft_vector_norm_workspace_bytes(n: int) -> int:
    return int(lib().deft_vector_norm_workspace_bytes(int(n)))


def deft_vector_norm(x, norm_d, ws, stream=None) -> None:
    _check("deft_vector_norm", lib().deft_vector_norm(_dp(x), x.numel(), _dp(norm_d), _dp(ws),
                                                      ws.numel() * ws.element_size(), _stream(stream)))


def deft_residual_update(acc, idx_d, count: int, stream=None) -> None:
    import torch
    if count > idx_d.numel():
        raise ValueError("count exceeds idx_d")
    _check("deft_residual_update",
           lib().deft_residual_update(_dp(acc, torch.float32), acc.numel(), _dp(idx_d, torch.int64), int(count),
                                      _stream(stream)))


def deft_topk_baseline(acc, k: int, val_d, idx_d, ws, stream=None) -> None:
    import torch
    if min(val_d.numel(), idx_d.numel()) < k:
        raise DeftError("deft_topk_baseline", ERR_CAPACITY)
    _check("deft_topk_baseline",
           lib().deft_topk_baseline(_dp(acc, torch.float32), acc.numel(), int(k), _dp(val_d, torch.float32),
                                    _dp(idx_d, torch.int64), _dp(ws), ws.numel() * ws.element_size(),
                                    _stream(stream)))


# ------------------------------------------------------------------------------------------
# row operators: embedding lookup, its gradient, dropout
# ------------------------------------------------------------------------------------------
F32, BF16, F16 = 0, 1, 2
MAX_PARTS = 8
EMBED_MAX_ROWS = 3000000
_TYPES = None


def _type(t) -> int:
    global _TYPES
    if _TYPES is None:
        import torch
        _TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
    code = _TYPES.get(t.dtype)
    if code is None:
        raise ValueError("expected float32, bfloat16 or float16, got %s" % t.dtype)
    return code


def _matrix(t, name: str) -> Tuple[int, int, int]:
    """(rows, columns, pitch) of a tensor whose last dimension is the row and whose others are one list of rows."""
    if t.dim() == 0:
        raise ValueError("%s: at least one dimension expected" % name)
    cols = t.size(-1)
    if t.is_contiguous():
        return (t.numel() // cols if cols else 0), cols, cols
    lead = [(n, s) for n, s in zip(t.shape[:-1], t.stride()[:-1]) if n != 1]
    if any(s0 != n1 * s1 for (_, s0), (n1, s1) in zip(lead, lead[1:])) or (cols > 1 and t.stride(-1) != 1):
        raise ValueError("%s: the rows must be contiguous and evenly spaced" % name)
    pitch = lead[-1][1] if lead else cols
    if pitch < cols:
        raise ValueError("%s: the rows overlap" % name)
    return t.numel() // cols, cols, pitch


def _device(first, *others) -> int:
    """The one CUDA device that the tensors (None: not given) lie on."""
    index = first.get_device()
    if index < 0:
        raise ValueError("expected CUDA tensors on one device")
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError("expected CUDA tensors on one device")
    return index


def _call(name: str, device: int, stream, *args) -> None:
    """Calls the library with `device` current, on `stream` or that device's current one."""
    import torch
    fn = getattr(_lib or lib(), name)
    handle = torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() == device:
        status = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            status = fn(*args, handle)
    if status:
        _check(name, status)


def _ids(ids) -> int:
    import torch
    if not ids.is_contiguous() or ids.dtype not in (torch.int64, torch.int32):
        raise ValueError("ids: a contiguous int64 or int32 tensor")
    return ids.element_size()


def _offset(offset_d) -> Optional[int]:
    if offset_d is None:
        return None
    import torch
    if offset_d.numel() != 1 or offset_d.dtype not in (torch.int64, torch.uint64):
        raise ValueError("offset_d: one 64-bit integer")
    return offset_d.data_ptr()


def _factor_fits(scale: float, p: float) -> bool:
    """Whether scale times the gain of the elements that dropout keeps is finite in fp32 (0 <= p < 1)."""
    x = scale * (65536.0 / (65536.0 - min(65535.0, math.floor(p * 65536.0 + 0.5))))
    return abs(x) < 2.0 ** 128 - 2.0 ** 103          # from there on the nearest fp32 number is an infinity


_U64 = (1 << 64) - 1


def deft_embed(table, ids, out, scale: float = 1.0, pos=None, p: float = 0.0, seed: int = 0, offset: int = 0,
               offset_d=None, stream=None) -> None:
    """out[t] = D(scale * table[ids[t]] + pos[t % len(pos)]), D = dropout (see deft_dropout)."""
    n, width, ld_out = _matrix(out, "out")
    if table.dim() != 2 or table.shape[1] != width or ids.numel() != n:
        raise ValueError("table, ids and out disagree")
    rows, _, ld_table = _matrix(table, "table")
    pos_rows = ld_pos = 0
    if pos is not None:
        pos_rows, w, ld_pos = _matrix(pos, "pos")
        if w != width or pos.dtype != table.dtype:
            raise ValueError("pos: rows like the table's expected")
    dev = _device(out, table, ids, pos, offset_d)
    _call("deft_embed", dev, stream, table.data_ptr(), _type(table), rows, width, ld_table, ids.data_ptr(), _ids(ids), n, scale,
          None if pos is None else pos.data_ptr(), pos_rows, ld_pos, p, seed & _U64, offset & _U64, _offset(offset_d), out.data_ptr(),
          _type(out), ld_out)


def deft_embed_workspace_bytes(n: int, rows: int, width: int) -> int:
    return int(lib().deft_embed_workspace_bytes(int(n), int(rows), int(width)))


def alloc_embed_workspace(n: int, rows: int, width: int, device="cuda"):
    """A torch uint8 tensor for deft_embed_grad calls of up to n tokens on a table of [rows, width]."""
    import torch
    size = deft_embed_workspace_bytes(n, rows, width)
    if size == 0:
        raise DeftError("deft_embed_workspace_bytes", ERR_INVALID_ARG)
    return torch.empty(size, dtype=torch.uint8, device=device)


def deft_embed_grad(grad_out, ids, grad, ws, accumulate: bool = False, skip_id: int = -1, scale: float = 1.0, p: float = 0.0,
                    seed: int = 0, offset: int = 0, offset_d=None, stream=None) -> None:
    """deft_embed's gradient with respect to the table, written to (or, with accumulate, added to the touched
    rows of) grad, a contiguous fp32 [rows, width] tensor: usually a view of the flat gradient vector or of the residual."""
    import torch
    if grad.dim() != 2 or not grad.is_contiguous() or grad.dtype != torch.float32:
        raise ValueError("grad: a contiguous float32 [rows, width] tensor")
    rows, width = grad.shape
    n, w, ld = _matrix(grad_out, "grad_out")
    if ids.numel() == 0 and grad_out.numel() == 0:
        n, w, ld = 0, width, width
    if w != width or ids.numel() != n:
        raise ValueError("grad_out, ids and grad disagree")
    if not ws.is_contiguous():
        raise ValueError("ws: a contiguous tensor")
    dev = _device(grad, grad_out, ids, ws, offset_d)
    _call("deft_embed_grad", dev, stream, grad_out.data_ptr(), _type(grad_out), ld, ids.data_ptr(), _ids(ids), n, rows, width, skip_id, scale, p,
          seed & _U64, offset & _U64, _offset(offset_d), grad.data_ptr(), 1 if accumulate else 0, ws.data_ptr(),
          ws.numel() * ws.element_size())


def deft_dropout(x, y, add=None, p: float = 0.5, seed: int = 0, offset: int = 0, offset_d=None, stream=None) -> None:
    """y = add + D(x) row by row (the last dimension is the row): kept elements times 1 / (1 - p), the mask a function
    of (seed, offset, row, column) alone.  The gradient is the same call on the incoming gradient without add."""
    rows, cols, ld_x = _matrix(x, "x")
    if y.shape != x.shape or (add is not None and (add.shape != x.shape or add.dtype != y.dtype)):
        raise ValueError("x, y and add disagree")
    ld_y = _matrix(y, "y")[2]
    ld_add = 0 if add is None else _matrix(add, "add")[2]
    dev = _device(y, x, add, offset_d)
    _call("deft_dropout", dev, stream, x.data_ptr(), _type(x), ld_x, None if add is None else add.data_ptr(), ld_add, y.data_ptr(), _type(y), ld_y,
          rows, cols, p, seed & _U64, offset & _U64, _offset(offset_d))


# ------------------------------------------------------------------------------------------
# dense row operators: layer norm and its gradient, rotary positions, distillation loss
# ------------------------------------------------------------------------------------------
NORM_MAX_COLS = 16384
DISTILL_MAX_VOCAB = 262144
DISTILL_MAX_TOP = 1024
ROTARY_MAX_ROT = 4096
_ROTARY_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3}


_FLOAT = None                      # torch.float32, once torch is there


def _vector(t, name: str, count: int, dtype=None) -> Optional[int]:
    """The pointer of a contiguous vector of `count` elements (None: not given); fp32 unless dtype says otherwise."""
    if t is None:
        return None
    if dtype is None:
        dtype = _FLOAT or _float()
    if t.numel() != count or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError("%s: a contiguous %s tensor of %d elements expected" % (name, dtype, count))
    return t.data_ptr()


def _float():
    global _FLOAT
    import torch
    _FLOAT = torch.float32
    return _FLOAT


def _like(t, name: str, shape, dtype, cols: int) -> Tuple[Optional[int], int]:
    """Pointer and pitch of a matrix of a given shape and type (None: not given)."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError("%s: a %s tensor of %s expected" % (name, dtype, tuple(shape)))
    return t.data_ptr(), cols if t.is_contiguous() else _matrix(t, name)[2]


def _weights(gamma, beta, cols: int) -> Tuple[Optional[int], Optional[int], int]:
    first = gamma if gamma is not None else beta
    if first is None:
        return None, None, F32
    dtype = first.dtype
    return _vector(gamma, "gamma", cols, dtype), _vector(beta, "beta", cols, dtype), _type(first)


def deft_layer_norm(x, y, gamma=None, beta=None, eps: float = 1e-5, add=None, sum=None, mean=None, rstd=None, stream=None) -> None:
    """y = layer norm of the rows (the last dimension) of x + add; the sum goes to `sum`, the statistics that the
    gradient needs to mean and rstd (fp32, one number per row)."""
    rows, cols, ld_x = _matrix(x, "x")
    shape, dtype = x.shape, x.dtype
    if y.shape != shape:
        raise ValueError("x and y disagree")
    ld_y = cols if y.is_contiguous() else _matrix(y, "y")[2]
    p_add, ld_add = _like(add, "add", shape, dtype, cols)
    p_sum, ld_sum = _like(sum, "sum", shape, dtype, cols)
    p_gamma, p_beta, w_type = _weights(gamma, beta, cols)
    dev = _device(y, x, add, sum, gamma, beta, mean, rstd)
    _call("deft_layer_norm", dev, stream, x.data_ptr(), _type(x), ld_x, p_add, ld_add, p_sum, ld_sum, p_gamma, p_beta, w_type, y.data_ptr(),
          _type(y), ld_y, rows, cols, eps, _vector(mean, "mean", rows), _vector(rstd, "rstd", rows))


def deft_layer_norm_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().deft_layer_norm_workspace_bytes(int(rows), int(cols)))


def alloc_layer_norm_workspace(rows: int, cols: int, device="cuda"):
    """A torch uint8 tensor for deft_layer_norm_grad calls of up to `rows` rows of up to `cols` columns."""
    import torch
    size = deft_layer_norm_workspace_bytes(rows, cols)
    if size == 0:
        raise DeftError("deft_layer_norm_workspace_bytes", ERR_INVALID_ARG)
    return torch.empty(size, dtype=torch.uint8, device=device)


def deft_layer_norm_grad(grad_out, x, mean, rstd, grad_x=None, gamma=None, add=None, grad_gamma=None, grad_beta=None, ws=None,
                         accumulate: bool = False, scale: float = 1.0, stream=None) -> None:
    """deft_layer_norm's gradient: with respect to x into grad_x (plus `add`, what reaches x past the norm), with respect to
    gamma and beta into grad_gamma and grad_beta, fp32 vectors (usually views of the flat gradient vector or of the
    residual), written, or with accumulate added to.  What is None is not computed."""
    rows, cols, ld_x = _matrix(x, "x")
    shape, dtype = x.shape, x.dtype
    if grad_out.shape != shape:
        raise ValueError("grad_out and x disagree")
    ld_go = cols if grad_out.is_contiguous() else _matrix(grad_out, "grad_out")[2]
    p_add, ld_add = _like(add, "add", shape, dtype, cols)
    p_gx, ld_gx = _like(grad_x, "grad_x", shape, dtype, cols)
    p_gamma, _, w_type = _weights(gamma, None, cols)
    if ws is not None and not ws.is_contiguous():
        raise ValueError("ws: a contiguous tensor")
    dev = _device(x, grad_out, mean, rstd, grad_x, gamma, add, grad_gamma, grad_beta, ws)
    _call("deft_layer_norm_grad", dev, stream, grad_out.data_ptr(), _type(grad_out), ld_go, x.data_ptr(), _type(x), ld_x, _vector(mean, "mean", rows),
          _vector(rstd, "rstd", rows), p_gamma, w_type, p_add, ld_add, p_gx, ld_gx, _vector(grad_gamma, "grad_gamma", cols),
          _vector(grad_beta, "grad_beta", cols), rows, cols, 1 if accumulate else 0, scale, None if ws is None else ws.data_ptr(),
          0 if ws is None else ws.numel() * ws.element_size())


def deft_rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, original: float = 0.0, low: float = 1.0,
                            high: float = 32.0) -> np.ndarray:
    """The frequencies of deft_rotary's rot / 2 pairs, an int64 array (the bits of unsigned fractions of a turn): base^(-2 i / rot) radians
    per position, stretched for contexts `factor` times as long ("linear", "base", or "parts": by their turns over the `original`
    context, kept from `high` turns on, stretched in full up to `low`)."""
    if scaling not in _ROTARY_SCALINGS:
        raise ValueError("scaling: one of %s" % ", ".join(_ROTARY_SCALINGS))
    out = np.zeros(max(1, int(rot) // 2), dtype=np.int64)
    if int(rot) <= ROTARY_MAX_ROT:
        _check("deft_rotary_frequencies", lib().deft_rotary_frequencies(int(rot), base, _ROTARY_SCALINGS[scaling], factor, original, low, high, _hp(out)))
    else:
        raise DeftError("deft_rotary_frequencies", ERR_TOO_LARGE)
    return out


_Strides = ctypes.c_int64 * 3


def _heads(t, name: str):
    """(batch, tokens, heads, dim) and the strides of a [batch, tokens, heads, dim] or [tokens, heads, dim] tensor."""
    strides = t.stride()
    if len(strides) == 4:
        b, n, h, d = t.shape
        sb, sn, sh, sd = strides
    elif len(strides) == 3:
        b, sb = 1, 0
        n, h, d = t.shape
        sn, sh, sd = strides
    else:
        raise ValueError("%s: a [batch, tokens, heads, dim] or [tokens, heads, dim] tensor" % name)
    if sd != 1 and d > 1:
        raise ValueError("%s: the columns of a head must be contiguous" % name)
    return b, n, h, d, _Strides(sb, sn, sh)


def deft_rotary(x, y, turns, positions=None, interleaved: bool = False, inverse: bool = False, gain: float = 1.0, stream=None) -> None:
    """Rotary positions: the first 2 len(turns) columns of every head of x ([batch, tokens, heads, dim] or [tokens, heads, dim], any
    strides of the first ones) turned by position times frequency; the others are copied.  y may be x.  turns:
    deft_rotary_frequencies on the device.  positions: int64 or int32, one per token (None: its number in its sequence).  inverse: the
    gradient with respect to x of the same call, applied to the gradient of y."""
    batch, tokens, heads, dim, xs = _heads(x, "x")
    if y.shape != x.shape or y.dtype is not x.dtype:
        raise ValueError("x and y disagree")
    ys = _heads(y, "y")[4]
    if turns.dim() != 1 or turns.element_size() != 8 or turns.is_floating_point() or turns.is_complex() or not turns.is_contiguous():
        raise ValueError("turns: a contiguous vector of 64-bit integers")
    p_pos, pos_bytes = None, 0
    if positions is not None:
        if positions.shape != x.shape[:-2]:
            raise ValueError("positions: one for each token expected")
        p_pos, pos_bytes = positions.data_ptr(), _ids(positions)
    dev = _device(y, x, turns, positions)
    _call("deft_rotary", dev, stream, x.data_ptr(), xs, y.data_ptr(), ys, _type(x), batch, tokens, heads, dim, turns.data_ptr(), 2 * turns.numel(),
          1 if interleaved else 0, 1 if inverse else 0, gain, p_pos, pos_bytes)


def deft_distill(logits, top_ids, top_logits, loss=None, grad=None, teacher_lse=None, temperature: float = 1.0, weight=None, scale: float = 1.0,
                 stream=None) -> None:
    """temperature^2 KL(teacher || student) of every row of logits (the last dimension is the vocabulary) into loss (fp32, one number per
    row) and scale times its gradient into grad (of the logits' type; may be the logits).  The teacher: its entries' ids and logits,
    renormalised over them, or with teacher_lse (its own log-sum-exp at the temperature, one number per row) with one class for
    all other tokens.  weight: fp32, one number per row; rows of weight 0 are not read."""
    rows, vocab, ld = _matrix(logits, "logits")
    shape, ids_shape = logits.shape, top_ids.shape
    if ids_shape != top_logits.shape or len(ids_shape) == 0 or ids_shape[:-1] != shape[:-1]:
        raise ValueError("logits, top_ids and top_logits disagree")
    if top_ids.is_floating_point() or top_ids.element_size() not in (4, 8) or not top_ids.is_signed() or top_ids.is_complex():
        raise ValueError("top_ids: an int64 or int32 tensor")
    top = ids_shape[-1]
    ld_ids = top if top_ids.is_contiguous() else _matrix(top_ids, "top_ids")[2]
    ld_teacher = top if top_logits.is_contiguous() else _matrix(top_logits, "top_logits")[2]
    p_grad, ld_grad = _like(grad, "grad", shape, logits.dtype, vocab)
    dev = _device(logits, top_ids, top_logits, loss, grad, teacher_lse, weight)
    _call("deft_distill", dev, stream, logits.data_ptr(), _type(logits), ld, rows, vocab, top_ids.data_ptr(), top_ids.element_size(), ld_ids,
          top_logits.data_ptr(), _type(top_logits), ld_teacher, top, _vector(teacher_lse, "teacher_lse", rows), temperature,
          _vector(weight, "weight", rows), scale, _vector(loss, "loss", rows), p_grad, ld_grad)
